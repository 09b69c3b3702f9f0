// Short causal depthwise convolution over packed sequences, with the kept tail of each sequence:
//
//   y[t][c] = act( sum_{j < K} w[c][j] * x~[t - (K - 1) + j][c] + bias[c] )
//
// where x~ before a sequence's first token is its tail, the last K - 1 rows that earlier calls saw.  The layer moves every
// element once and does K multiply-adds with it: memory bounds it, and the launch itself for single tokens.  A thread owns
// 16 bytes of a row (its channels' taps stay in registers) and a run of tokens, over which it slides a window of rows, four
// rows loaded at a time; K - 1 rows of a run are read twice.  8192 x 4096, K = 4, SiLU, three sets of tensors in turn: fp16 33.5 us, 4.0 TB/s, fp32
// 47 us, 5.7 TB/s (a large copy: 5.1 to 5.5); element by element, where rows are not 16-byte aligned, fp16 36 us.
#include <algorithm>
#include <type_traits>

#include "q4.h"
#include "sequence.h"

namespace cadnn {

namespace {

constexpr int kConvMaxTaps = 8;

struct CcArgs {
    const void* x;
    void* y;
    const float* w;       // [channels][K]
    const float* bias;
    void* state;          // [seqs][K - 1][channels] or NULL
    int64_t x_stride, y_stride;
    Sequences q;
    int channels, chunk, act, tx_log;
    int64_t slots, slot0;
};

template <typename T, int V, int K>
__global__ __launch_bounds__(256) void causal_conv_kernel(const CcArgs a) {
    typedef T VT __attribute__((ext_vector_type(V)));
    constexpr int U = 4;
    const int tx = (int)threadIdx.x & ((1 << a.tx_log) - 1);
    const int64_t slot = a.slot0 + (int64_t)blockIdx.x * (256 >> a.tx_log) + ((int)threadIdx.x >> a.tx_log);
    const int c = ((int)blockIdx.y * (1 << a.tx_log) + tx) * V;
    if (slot >= a.slots || c >= a.channels) return;
    int piece, lo, hi;
    const int s = seq_of_slot(a.q, (int)slot, a.chunk, &piece);
    seq_range(a.q, s, &lo, &hi);
    const int64_t first = lo + (int64_t)piece * a.chunk;
    if (piece < 0 || first >= hi) return;
    const int t0 = (int)first, t1 = (int)min((int64_t)hi, first + a.chunk);
    const T* x = (const T*)a.x + c;
    T* y = (T*)a.y + c;
    T* tail = a.state ? (T*)a.state + ((int64_t)s * (K - 1)) * a.channels + c : nullptr;
    float w[V][K], b[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
        for (int k = 0; k < K; ++k) w[v][k] = a.w[(int64_t)(c + v) * K + k];
        b[v] = a.bias ? a.bias[c + v] : 0.0f;
    }
    VT row[K - 1 + U];
    // the rows before the run
    const VT zero = (VT)(T)0.0f;
#pragma unroll
    for (int r = 0; r < K - 1; ++r) {
        const int t = t0 - (K - 1) + r;
        row[r] = t >= lo ? *(const VT*)(x + (int64_t)t * a.x_stride)
                         : tail ? *(const VT*)(tail + (int64_t)(t - lo + K - 1) * a.channels) : zero;
    }
    if (K > 1 && piece == 0 && tail) {
        // the new tail: this thread alone reads and writes its channels' old one
        VT last[K > 1 ? K - 1 : 1];
#pragma unroll
        for (int r = 0; r < K - 1; ++r) {
            const int t = hi - (K - 1) + r;
            last[r] = t >= lo ? *(const VT*)(x + (int64_t)t * a.x_stride) : *(const VT*)(tail + (int64_t)(t - lo + K - 1) * a.channels);
        }
#pragma unroll
        for (int r = 0; r < K - 1; ++r) *(VT*)(tail + (int64_t)r * a.channels) = last[r];
    }
    // A tap that is exactly zero is not applied, whatever it would meet; a wave without one does not look.
    bool zeros = false;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int k = 0; k < K; ++k) zeros |= w[v][k] == 0.0f;
    // (four rows are worked on while the next four are on their way)
    VT ahead[U];
    auto fetch = [&](int t) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            ahead[u] = zero;
            if (t + u < t1) ahead[u] = *(const VT*)(x + (int64_t)(t + u) * a.x_stride);
        }
    };
    fetch(t0);
    // (the activation is settled outside the loop: a branch for each element would part them from each other, 37 us at 8192 x 4096, fp16)
    auto run = [&](auto skip, auto act) {
        for (int t = t0; t < t1; t += U) {
#pragma unroll
            for (int u = 0; u < U; ++u) row[K - 1 + u] = ahead[u];
            if (t + U < t1) fetch(t + U);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                VT out;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    float acc = b[v];
#pragma unroll
                    for (int k = 0; k < K; ++k) acc = !skip.value || w[v][k] != 0.0f ? fmaf(w[v][k], (float)row[u + k][v], acc) : acc;
                    out[v] = (T)apply_act(acc, act.value < 0 ? a.act : act.value);
                }
                if (t + u < t1) *(VT*)(y + (int64_t)(t + u) * a.y_stride) = out;
            }
#pragma unroll
            for (int r = 0; r < K - 1; ++r) row[r] = row[r + U];
        }
    };
    if (__any(zeros)) run(std::true_type{}, std::integral_constant<int, -1>{});
    else if (a.act == CADNN_ACT_SILU) run(std::false_type{}, std::integral_constant<int, CADNN_ACT_SILU>{});
    else if (a.act == CADNN_ACT_RELU) run(std::false_type{}, std::integral_constant<int, CADNN_ACT_RELU>{});
    else run(std::false_type{}, std::integral_constant<int, CADNN_ACT_NONE>{});
}

template <typename T, int V, int K>
hipError_t launch_cc(CcArgs a, hipStream_t s) {
    const int vectors = (a.channels + V - 1) / V, tx = 1 << a.tx_log, per = 256 / tx;
    const int64_t blocks = (a.slots + per - 1) / per, step = 1 << 23;      // (a launch has fewer than 2^32 threads to a row of workgroups)
    for (int64_t b = 0; b < blocks; b += step) {
        a.slot0 = b * per;
        const dim3 grid((unsigned)std::min(step, blocks - b), (unsigned)((vectors + tx - 1) / tx));
        CADNN_LAUNCH((causal_conv_kernel<T, V, K>), grid, dim3(256), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T, int V>
hipError_t launch_cc_taps(CcArgs a, int taps, hipStream_t s) {
    const int vectors = (a.channels + V - 1) / V;
    a.tx_log = 0;
    while (a.tx_log < 8 && (1 << a.tx_log) < vectors) ++a.tx_log;
    // The longest run that still leaves 131072 threads (eight waves to a compute unit): a run of 64 tokens reads 5 % of
    // the rows twice at K = 4, one of 8 tokens 38 %.  (8192 x 4096, fp16: 131072 threads 37.4 us, twice as many 40.0.)
    a.chunk = 64;
    while (a.chunk > 8 && seq_slots(a.q.tokens, a.q.seqs, a.q.start != nullptr, a.chunk) * vectors < 131072) a.chunk /= 2;
    a.slots = seq_slots(a.q.tokens, a.q.seqs, a.q.start != nullptr, a.chunk);
    switch (taps) {
        case 1: return launch_cc<T, V, 1>(a, s);
        case 2: return launch_cc<T, V, 2>(a, s);
        case 3: return launch_cc<T, V, 3>(a, s);
        case 4: return launch_cc<T, V, 4>(a, s);
        case 5: return launch_cc<T, V, 5>(a, s);
        case 6: return launch_cc<T, V, 6>(a, s);
        case 7: return launch_cc<T, V, 7>(a, s);
        default: return launch_cc<T, V, 8>(a, s);
    }
}

template <typename T>
hipError_t launch_cc_type(const CcArgs& a, int taps, hipStream_t s) {
    constexpr int V = 16 / (int)sizeof(T);
    const int64_t e = sizeof(T);
    const bool vec = a.channels % V == 0 && (uintptr_t)a.x % 16 == 0 && (uintptr_t)a.y % 16 == 0 && (uintptr_t)a.state % 16 == 0 &&
                     a.x_stride * e % 16 == 0 && a.y_stride * e % 16 == 0;
    return vec ? launch_cc_taps<T, V>(a, taps, s) : launch_cc_taps<T, 1>(a, taps, s);
}

}  // namespace

cadnn_status check_sequences(const char* who, int tokens, int seqs, const int32_t* seq_start) {
    if (tokens < 0 || seqs <= 0) return fail(CADNN_EINVAL, "%s: a negative number of tokens or no sequence", who);
    if (seqs > (1 << 24) || tokens > (1 << 30)) return fail(CADNN_EUNSUPPORTED, "%s: more than 2^24 sequences or 2^30 tokens", who);
    if ((uintptr_t)seq_start % 4) return fail(CADNN_EINVAL, "%s: seq_start is misaligned", who);
    if (!seq_start && tokens % seqs) return fail(CADNN_EINVAL, "%s: %d tokens are not %d sequences of one length", who, tokens, seqs);
    return CADNN_OK;
}

}  // namespace cadnn

using namespace cadnn;

extern "C" cadnn_status cadnn_causal_conv1d(const cadnn_weights* w, const void* x, int64_t x_stride, void* y, int64_t y_stride,
                                            int tokens, int seqs, const int32_t* seq_start, void* state, const void* bias,
                                            int act, void* stream) {
    const char* who = "cadnn_causal_conv1d";
    if (!w) return fail(CADNN_EINVAL, "%s: NULL handle", who);
    if (w->cin != 1 || w->kh != 1) return fail(CADNN_EINVAL, "%s: weights are [%d][%d][%d][%d], not [channels][1][1][taps]", who, w->cout, w->cin, w->kh, w->kw);
    if (w->kw > kConvMaxTaps) return fail(CADNN_EUNSUPPORTED, "%s: %d taps (at most %d are served)", who, w->kw, kConvMaxTaps);
    if (w->cout > (1 << 23)) return fail(CADNN_EUNSUPPORTED, "%s: more than 2^23 channels", who);
    cadnn_status st = check_sequences(who, tokens, seqs, seq_start);
    if (st != CADNN_OK) return st;
    if (act != CADNN_ACT_NONE && act != CADNN_ACT_RELU && act != CADNN_ACT_SILU) return fail(CADNN_EINVAL, "%s: unknown activation %d", who, act);
    if (tokens == 0) return CADNN_OK;
    if (!x || !y) return fail(CADNN_EINVAL, "%s: NULL tensor", who);
    if (x == y || state == x || state == y) return fail(CADNN_EINVAL, "%s: x, y and state must not overlap", who);
    if (x_stride < w->cout || y_stride < w->cout) return fail(CADNN_EINVAL, "%s: rows overlap (a stride below the number of channels)", who);
    const size_t e = w->elem();
    if ((uintptr_t)x % e || (uintptr_t)y % e || (uintptr_t)state % e || (uintptr_t)bias % 4) return fail(CADNN_EINVAL, "%s: a misaligned pointer", who);
    bool ready;
    {
        std::lock_guard<std::mutex> lock(w->mu);
        ready = w->dw_ready;
    }
    if (!ready) {
        hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
        CADNN_HIP(hipStreamIsCapturing((hipStream_t)stream, &cap));
        if (cap != hipStreamCaptureStatusNone)
            return fail(CADNN_EINVAL, "%s: the first call uploads the weights and cannot be captured (cadnn_depthwise_prepare)", who);
    }
    if ((st = ensure_dw_device(w)) != CADNN_OK) return st;
    int device = -1;
    CADNN_HIP(hipGetDevice(&device));
    if (device != w->dw_device) return fail(CADNN_EINVAL, "%s: the weights are on device %d, the current one is %d", who, w->dw_device, device);
    CcArgs a{};
    a.x = x; a.y = y; a.w = (const float*)w->d_dw.p; a.bias = (const float*)bias; a.state = w->kw > 1 ? state : nullptr;
    a.x_stride = x_stride; a.y_stride = y_stride;
    a.q = Sequences{seq_start, tokens, seqs};
    a.channels = w->cout; a.act = act;
    CADNN_HIP(w->dtype == CADNN_F16 ? launch_cc_type<_Float16>(a, w->kw, (hipStream_t)stream)
                                    : launch_cc_type<float>(a, w->kw, (hipStream_t)stream));
    return CADNN_OK;
}
