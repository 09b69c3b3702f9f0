// Selective state space scan over packed sequences.  For every token t, channel c and state n
//
//   dt = dt_raw[t][c] + dt_bias[c], through softplus if asked
//   h[c][n] = exp(dt * a[c][n]) * h[c][n] + dt * x[t][c] * b[t][g(c)][n]
//   y[t][c] = (sum_n c[t][g(c)][n] * h[c][n] + d[c] * x[t][c]) * silu(z[t][c])
//
// Every (t, c, n) costs an exponential (half the vector rate, measured) and four full-rate operations, some 24 cycles of a
// SIMD per 64 of them, against 4 / N elements of traffic: from N = 16 on the vector units bound a long scan, and the
// states' traffic a single token.  A long sequence is a chain of tokens that only channels and states run beside, so it is cut into
// pieces: one pass for what each piece ends with, a join, one for the outputs -- the exponentials are taken twice.  us at 4096
// tokens x 2048 channels x 16 states, gated, fp16: 30 + 11 + 38 (four waves a SIMD; 20 for the vector work of one pass at its rate, 12 for the
// traffic); one token of 64 sequences x 4096 x 16: 10.4, 3.5 TB/s.
#include <type_traits>

#include "q4.h"
#include "sequence.h"

namespace cadnn {

namespace {

constexpr int kScanMaxStates = 256;
constexpr int kScanTile = 8;          // tokens whose inputs are fetched together

struct SsArgs {
    const void *x, *dt, *b, *c, *z;
    void* y;
    int64_t x_stride, dt_stride, b_stride, c_stride, z_stride, y_stride;
    const float *a, *d, *dt_bias;
    float* state;         // [seqs][channels][dstate] or NULL
    float* part;          // pieces: [slot][channels][dstate], the piece's own end state, later the state it starts from
    float* span;          // pieces: [slot][channels], the sum of the time steps
    Sequences q;
    int channels, dstate, groups, per, softplus;
    int chunk, blocks_per_group, longest;
    int64_t slots;
};

__device__ __forceinline__ float ss_exp2(float v) { return __builtin_amdgcn_exp2f(v); }

// step * log2(e), for exp(step * a) = exp2(step * log2(e) * a): a stays as it is, so that a step of zero keeps the state whatever finite value a has.
__device__ __forceinline__ float ss_base2(float step) { return step * 1.44269502f; }

// log(1 + exp(v)) = max(v, 0) + log1p(e), e = exp(-|v|), from the product |v| * log2(e) in two parts.  log1p(e) = e + e^2 q(e), whose q of
// degree 8 was fitted to it for 0 <= e <= 1 (relative error 2^-27, 1.4 * 2^-24 with the roundings of its evaluation).
__device__ __forceinline__ float ss_softplus(float v) {
    const float m = fminf(fabsf(v), 150.0f);      // (exp is zero from there on; the two parts of an infinity would be no numbers)
    const float hi = m * -1.44269502f, lo = fmaf(m, -1.92596303e-8f, fmaf(m, -1.44269502f, -hi));
    const float e = ss_exp2(hi) * fmaf(lo, 0.693147182f, 1.0f);
    float q = -0.00324401166f;
    q = fmaf(q, e, 0.0198514052f);
    q = fmaf(q, e, -0.0569594353f);
    q = fmaf(q, e, 0.106036462f);
    q = fmaf(q, e, -0.153055876f);
    q = fmaf(q, e, 0.196759388f);
    q = fmaf(q, e, -0.249541342f);
    q = fmaf(q, e, 0.333299637f);
    q = fmaf(q, e, -0.499999017f);
    return (v < 0.0f ? 0.0f : v) + fmaf(q * e, e, e);      // (no number stays none)
}

// The gate.  fp32 storage: to 6 half steps.  fp16: the exponent is rounded once, an error of 3 |v| half steps of fp32, which fp16's own half step hides (2^-11 to
// 3 * 21 * 2^-24 where the gate is not zero in fp16); 4096 tokens x 2048 channels x 16 states take 78.1 us so, 79.1 with the other.
template <typename T>
__device__ __forceinline__ float ss_silu(float v) {
    if constexpr (sizeof(T) == 4) return act_silu(v);
    return v * __builtin_amdgcn_rcpf(1.0f + ss_exp2(v * -1.44269502f));
}

// Sum over the L consecutive lanes that share a channel.
template <int L>
__device__ __forceinline__ float ss_sum(float v) {
    if constexpr (L >= 2) v += __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0xB1, 0xf, 0xf, true));     // lane ^ 1
    if constexpr (L >= 4) v += __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0x4E, 0xf, 0xf, true));     // lane ^ 2
    if constexpr (L >= 8) v += __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0x141, 0xf, 0xf, true));    // mirrored in 8 lanes
    if constexpr (L >= 16) v += __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0x140, 0xf, 0xf, true));   // mirrored in 16 lanes
    if constexpr (L >= 32) v += __shfl_xor(v, 16, 64);
    if constexpr (L >= 64) v += __shfl_xor(v, 32, 64);
    return v;
}

// f of eight values that four neighbouring lanes all hold: lane q takes values q and 4 + q, and passes them on.
// (softplus and silu of steps and gates took a tenth of the time where four lanes of a channel each worked out all of them: 1501 tokens x 1000
// channels x 64 states, fp32, passes 37.3 + 45.0 us, so 34.0 + 40.1; with log1p as a polynomial and one branch a tile 33.7 + 38.1)
template <typename F>
__device__ __forceinline__ void ss_shared(float (&v)[8], int sub, F f) {
    const int q = sub & 3;
#pragma unroll
    for (int k = 0; k < 8; k += 4) {
        const float own = f(q == 0 ? v[k] : q == 1 ? v[k + 1] : q == 2 ? v[k + 2] : v[k + 3]);
        const int bits = (int)__float_as_uint(own);
        v[k] = __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp(bits, 0x00, 0xf, 0xf, true));
        v[k + 1] = __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp(bits, 0x55, 0xf, 0xf, true));
        v[k + 2] = __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp(bits, 0xaa, 0xf, 0xf, true));
        v[k + 3] = __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp(bits, 0xff, 0xf, 0xf, true));
    }
}

// NS consecutive floats of a lane, `left` of which exist; 16 bytes at a time where all do (4-byte alignment is enough).
template <int NS>
__device__ __forceinline__ void ss_load(const float* p, int left, float (&v)[NS]) {
    typedef float F4 __attribute__((ext_vector_type(4), aligned(4)));
    if (left >= NS) {
#pragma unroll
        for (int k = 0; k < NS; k += 4) {
            const F4 q = *(const F4*)(p + k);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[k + e] = q[e];
        }
    } else {
#pragma unroll
        for (int k = 0; k < NS; ++k) v[k] = k < left ? p[k] : 0.0f;
    }
}
template <int NS>
__device__ __forceinline__ void ss_store(float* p, int left, const float (&v)[NS]) {
    typedef float F4 __attribute__((ext_vector_type(4), aligned(4)));
    if (left >= NS) {
#pragma unroll
        for (int k = 0; k < NS; k += 4) *(F4*)(p + k) = (F4){v[k], v[k + 1], v[k + 2], v[k + 3]};
    } else {
#pragma unroll
        for (int k = 0; k < NS; ++k)
            if (k < left) p[k] = v[k];
    }
}

enum ScanPass {
    SCAN_WHOLE,     // one pass over whole sequences
    SCAN_ENDS,      // of every piece: the state it ends with when it starts from zero
    SCAN_PIECES     // of every piece: its outputs, from the state it starts from
};

// L lanes hold a channel's states, NS each.  The inputs of kScanTile tokens are fetched while the tile before them is
// worked on; b and c, which all channels of a group share, go through LDS.  FULL: dstate = NS * L; else the
// states behind the last one stay zero whatever x and dt are.
template <typename T, int NS, int L, int PASS, bool FULL>
__global__ __launch_bounds__(256) void scan_kernel(const SsArgs a) {
    constexpr int CH = 256 / L, N = NS * L, TT = kScanTile;
    static_assert(TT == 8, "ss_shared");
    constexpr int ROW = PASS == SCAN_ENDS ? N : 2 * N;          // elements of a token in LDS
    constexpr int PER = (TT * ROW + 255) / 256;                 // of them fetched by a thread
    constexpr int V = 16 / (int)sizeof(T);
    typedef T VT __attribute__((ext_vector_type(V)));
    __shared__ __attribute__((aligned(16))) T bc[2][TT * ROW];
    const int tid = (int)threadIdx.x, sub = tid % L;
    const int grp = (int)blockIdx.y / a.blocks_per_group;
    const int in_group = ((int)blockIdx.y - grp * a.blocks_per_group) * CH + tid / L;
    const bool real = in_group < a.per;
    const int ch = grp * a.per + (real ? in_group : a.per - 1);
    int s, lo, hi, t0, t1;
    const int64_t slot = blockIdx.x;
    if (PASS == SCAN_WHOLE) {
        s = (int)slot;
        seq_range(a.q, s, &lo, &hi);
        t0 = lo;
        t1 = hi;
    } else {
        int piece;
        s = seq_of_slot(a.q, (int)slot, a.chunk, &piece);
        seq_range(a.q, s, &lo, &hi);
        const int64_t first = lo + (int64_t)piece * a.chunk;
        if (piece < 0 || first >= hi) return;
        t0 = (int)first;
        t1 = (int)min((int64_t)hi, first + a.chunk);
    }
    if (t0 >= t1) return;
    const uint32_t lane_bytes = (uint32_t)ch * (uint32_t)sizeof(T);
    // Rows are uniform, channels are the lanes': a scalar base and a 32-bit offset address a load.  (The compiler keeps them so if it does not see
    // what they are made of; else it adds them up for every lane, 96 instructions a tile.)
    typedef __attribute__((address_space(1))) char Global;
    auto here = [&]() -> uint32_t { uint32_t v = lane_bytes; asm volatile("" : "+v"(v)); return v; };
    auto at_row = [&](const void* base, int64_t stride, int at, uint32_t lane) -> __attribute__((address_space(1))) T* {
        Global* row = (Global*)((const char*)base + at * stride * (int64_t)sizeof(T));
        asm volatile("" : "+s"(row));
        return (__attribute__((address_space(1))) T*)(row + lane);
    };
    const T* bp = (const T*)a.b + (int64_t)grp * a.dstate;
    const T* cp = (const T*)a.c + (int64_t)grp * a.dstate;
    T nx[TT], nd[TT], nz[TT];
    T nb[PER];
#pragma unroll
    for (int u = 0; u < TT; ++u) nz[u] = (T)0.0f;
    // rows t to t + 7, and rows that lie in front of the sequence as its first one
    auto fetch = [&](int t, auto whole) {
        const uint32_t lane = here();
        auto row = [&](const void* base, int64_t stride, int u) -> T { return *at_row(base, stride, decltype(whole)::value ? t + u : max(t + u, t0), lane); };
#pragma unroll
        for (int u = 0; u < TT; ++u) nx[u] = row(a.x, a.x_stride, u);
#pragma unroll
        for (int u = 0; u < TT; ++u) nd[u] = row(a.dt, a.dt_stride, u);
        if (PASS != SCAN_ENDS && a.z) {
#pragma unroll
            for (int u = 0; u < TT; ++u) nz[u] = row(a.z, a.z_stride, u);
        }
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int i = k * 256 + tid, u = i / ROW, r = i % ROW, n = r < N ? r : r - N, at = t + u;
            T v = (T)0.0f;
            if (i < TT * ROW && (decltype(whole)::value || at >= t0) && (FULL || n < a.dstate))
                v = r < N ? bp[(int64_t)at * a.b_stride + n] : cp[(int64_t)at * a.c_stride + n];
            nb[k] = v;
        }
    };
    const bool has_whole = t1 - t0 >= TT;
    if (has_whole) fetch(t0, std::true_type{});
    else fetch(t1 - TT, std::false_type{});
    float h[NS], rate[NS];
    const int n_left = a.dstate - sub * NS;
    float* kept = nullptr;
    if (PASS == SCAN_WHOLE) kept = a.state ? a.state + ((int64_t)s * a.channels + ch) * a.dstate + sub * NS : nullptr;
    else kept = a.part + (slot * a.channels + ch) * a.dstate + sub * NS;
    ss_load<NS>(a.a + (int64_t)ch * a.dstate + sub * NS, FULL ? NS : n_left, rate);
    if (PASS != SCAN_ENDS && kept) ss_load<NS>(kept, FULL ? NS : n_left, h);
    else {
#pragma unroll
        for (int k = 0; k < NS; ++k) h[k] = 0.0f;
    }
    const float bias = a.dt_bias ? a.dt_bias[ch] : 0.0f;
    const float dv = a.d ? a.d[ch] : 0.0f;
    float span = 0.0f;
    int buf = 0;
    // The rows t to t + 7 that were fetched; of the last tile, where the sequence does not end with a whole one, they are the
    // sequence's last eight, and the first `skip` of them are done or in front of it.
    auto tile = [&](int t, int skip, auto whole) {
        constexpr bool W = decltype(whole)::value;
        float x[TT], dt[TT], z[TT];
#pragma unroll
        for (int u = 0; u < TT; ++u) {
            x[u] = (float)nx[u];
            dt[u] = (float)nd[u];
            if (PASS != SCAN_ENDS) z[u] = (float)nz[u];
        }
        // (converted here: put off, the conversions would have the next rows' loads write to other registers, and 24 copies)
#pragma unroll
        for (int u = 0; u < TT; ++u) {
            asm volatile("" : "+v"(x[u]), "+v"(dt[u]));
            if (PASS != SCAN_ENDS) asm volatile("" : "+v"(z[u]));
        }
#pragma unroll
        for (int k = 0; k < PER; ++k)
            if (k * 256 + tid < TT * ROW) bc[buf][k * 256 + tid] = nb[k];
        __syncthreads();     // (the other buffer is written next, after the next barrier's readers of this one)
        if (W) fetch(min(t + TT, t1 - TT), std::true_type{});      // (the last one's rows again where nothing follows: no branch parts the tile)
        float steps = 0.0f;          // (summed by tiles: 8 + chunk / 8 roundings at most, not chunk)
#pragma unroll
        for (int u = 0; u < TT; ++u) dt[u] += bias;
        // (one branch for the tile's tokens, whose chains of operations then run beside each other)
        if (a.softplus) {
            if constexpr (L >= 4) ss_shared(dt, sub, [](float v) { return ss_softplus(v); });
            else {
#pragma unroll
                for (int u = 0; u < TT; ++u) dt[u] = ss_softplus(dt[u]);
            }
        }
        if (PASS != SCAN_ENDS && a.z) {
            if constexpr (L >= 4) ss_shared(z, sub, [](float v) { return ss_silu<T>(v); });
            else {
#pragma unroll
                for (int u = 0; u < TT; ++u) z[u] = ss_silu<T>(z[u]);
            }
        }
        if (PASS == SCAN_ENDS) {
#pragma unroll
            for (int u = 0; u < TT; ++u) steps += W || u >= skip ? dt[u] : 0.0f;
            span += steps;
        }
        float ys[TT];
        // (outputs are stored behind the tile: a store under a condition would part the tokens' work from each other)
        // one token: three full-rate operations a state beside the exponential and the product under it
        auto token = [&](int u) {
            const float step = ss_base2(dt[u]), in = dt[u] * x[u];
            const T* row = bc[buf] + u * ROW + sub * NS;
            float y = 0.0f;
#pragma unroll
            for (int k0 = 0; k0 < NS; k0 += V) {
                const VT bv = *(const VT*)(row + k0);
                VT cv = bv;
                if (PASS != SCAN_ENDS) cv = *(const VT*)(row + N + k0);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const int k = k0 + e;
                    h[k] = fmaf((float)bv[e], in, ss_exp2(step * rate[k]) * h[k]);
                    if (!FULL) h[k] = sub * NS + k < a.dstate ? h[k] : 0.0f;
                    if (PASS != SCAN_ENDS) y = fmaf((float)cv[e], h[k], y);
                }
            }
            ys[u] = y;
        };
#pragma unroll
        for (int u = 0; u < TT; ++u) {
            if (!W) ys[u] = 0.0f;
            if (W || u >= skip) token(u);
        }
        if (PASS != SCAN_ENDS) {
#pragma unroll
            for (int u = 0; u < TT; ++u) ys[u] = fmaf(dv, x[u], ss_sum<L>(ys[u]));
            if (a.z) {
#pragma unroll
                for (int u = 0; u < TT; ++u) ys[u] *= z[u];
            }
            if (sub == 0 && real) {
                const uint32_t lane = here();
#pragma unroll
                for (int u = 0; u < TT; ++u)
                    if (W || u >= skip) *at_row(a.y, a.y_stride, t + u, lane) = (T)ys[u];
            }
        }
        buf ^= 1;
    };
    int t = t0;
    for (; t + TT <= t1; t += TT) tile(t, 0, std::true_type{});
    if (t < t1) tile(t1 - TT, TT - (t1 - t), std::false_type{});
    if (real && kept && PASS != SCAN_PIECES) {
        ss_store<NS>(kept, FULL ? NS : n_left, h);
        if (PASS == SCAN_ENDS && sub == 0) a.span[slot * a.channels + ch] = span;
    }
}

// 2^e as m * 2^n, for what a piece's steps, whose exponents add up to e, make of a state: 2^e itself may pass what fp32 holds, or vanish, where the
// state's product with it does neither.  m lies between 1/2 and 2, so that a state of zero stays zero and an infinite one infinite, as after any number of
// steps that each shrink it a little.  (Beyond 277 every product is zero or infinite.  Where e is no number, what the piece ends with is none either.)
struct SsFactor {
    float m;
    int n;
};
__device__ __forceinline__ SsFactor ss_factor(float e) {
    e = __builtin_amdgcn_fmed3f(e, -400.0f, 400.0f);
    const float n = truncf(e);
    return {ss_exp2(e - n), (int)n};
}

// What a piece ends with that starts from h and, from zero, ends with `end`.
__device__ __forceinline__ float ss_after(SsFactor f, float h, float end) { return __builtin_amdgcn_ldexpf(f.m * h, f.n) + end; }

// Joins the pieces of each sequence, h = exp(a * span) * h + end; what a piece ended with is replaced by what it starts from.
// A workgroup owns 64 (channel, state) pairs of a sequence.  Its four waves fetch S pieces each, join them from zero, learn
// from each other what they start from, and go through them again, in registers: the chain of a long sequence costs one
// round trip to memory for 4 * S pieces.  (64 pieces of 32768 pairs: 12.5 us with one thread for a pair's whole chain, 9.8 with S = 32, 6.6 with S = 16.)
template <int S>
__device__ __forceinline__ float ss_join(const SsArgs& a, int64_t per_seq, int64_t i, int ch, int64_t first, int p0, int pieces, float rate, float h, float (&lds)[2][4][64]) {
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    float end[S], span[S];
#pragma unroll
    for (int u = 0; u < S; ++u) {
        const int p = p0 + wave * S + u;
        const int64_t slot = first + min(p, pieces - 1);
        const bool there = p < pieces && slot < a.slots;
        end[u] = there ? a.part[slot * per_seq + i] : 0.0f;
        span[u] = there ? a.span[slot * a.channels + ch] : 0.0f;
    }
    SsFactor f[S];
    float all = 0.0f, own = 0.0f;       // of the wave's pieces together: steps are added up, as the product of factors could pass fp32 on its way
#pragma unroll
    for (int u = 0; u < S; ++u) {
        f[u] = ss_factor(rate * ss_base2(span[u]));
        own = ss_after(f[u], own, end[u]);
        all += span[u];
    }
    lds[0][wave][lane] = all;
    lds[1][wave][lane] = own;
    __syncthreads();
    float mine = h;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (w == wave) mine = h;
        h = ss_after(ss_factor(rate * ss_base2(lds[0][w][lane])), h, lds[1][w][lane]);
    }
#pragma unroll
    for (int u = 0; u < S; ++u) {
        const int p = p0 + wave * S + u;
        if (p < pieces && first + p < a.slots) a.part[(first + p) * per_seq + i] = mine;
        mine = ss_after(f[u], mine, end[u]);
    }
    __syncthreads();
    return h;
}

__global__ __launch_bounds__(256) void scan_join_kernel(const SsArgs a) {
    __shared__ float lds[2][4][64];
    const int64_t per_seq = (int64_t)a.channels * a.dstate, at = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
    const int64_t i = min(at, per_seq - 1);      // (lanes behind the last pair repeat it: same reads before, same values written)
    const int s = (int)blockIdx.y;
    int lo, hi;
    seq_range(a.q, s, &lo, &hi);
    if (lo >= hi) return;
    const int ch = (int)(i / a.dstate);
    const int64_t first = seq_first_slot(a.q, s, a.chunk);
    const int pieces = (int)(((int64_t)hi - lo + a.chunk - 1) / a.chunk);
    const float rate = a.a[i];
    float* kept = a.state ? a.state + (int64_t)s * per_seq + i : nullptr;
    float h = kept ? *kept : 0.0f;
    int p = 0;
    for (; pieces - p > 64; p += 128) h = ss_join<32>(a, per_seq, i, ch, first, p, pieces, rate, h, lds);
    for (; pieces - p > 32; p += 64) h = ss_join<16>(a, per_seq, i, ch, first, p, pieces, rate, h, lds);
    for (; p < pieces; p += 32) h = ss_join<8>(a, per_seq, i, ch, first, p, pieces, rate, h, lds);
    if (kept && at < per_seq && threadIdx.x < 64) *kept = h;
}

// The same for sequences of few pieces: one thread for a pair's whole chain, four pieces fetched at a time.
__global__ __launch_bounds__(256) void scan_join_few_kernel(const SsArgs a) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, per_seq = (int64_t)a.channels * a.dstate;
    if (i >= per_seq) return;
    const int s = (int)blockIdx.y;
    int lo, hi;
    seq_range(a.q, s, &lo, &hi);
    if (lo >= hi) return;
    const int ch = (int)(i / a.dstate);
    const int64_t first = seq_first_slot(a.q, s, a.chunk);
    const int pieces = (int)min(((int64_t)hi - lo + a.chunk - 1) / a.chunk, a.slots - first);
    const float rate = a.a[i];
    float* kept = a.state ? a.state + (int64_t)s * per_seq + i : nullptr;
    float h = kept ? *kept : 0.0f;
    float* part = a.part + first * per_seq + i;
    const float* span = a.span + first * a.channels + ch;
    constexpr int U = 4;
    for (int p = 0; p < pieces; p += U) {
        float end[U] = {}, steps[U] = {};
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (p + u < pieces) {
                end[u] = part[u * per_seq];
                steps[u] = span[(int64_t)u * a.channels];
            }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (p + u < pieces) {
                part[u * per_seq] = h;
                h = ss_after(ss_factor(rate * ss_base2(steps[u])), h, end[u]);
            }
        part += U * per_seq;
        span += (int64_t)U * a.channels;
    }
    if (kept) *kept = h;
}

// Few tokens a sequence: L lanes hold a channel's states, four each, so that a wave reads and writes them in whole
// kilobytes; b and c come straight from memory.
template <typename T, int L>
__global__ __launch_bounds__(256) void scan_few_kernel(const SsArgs a) {
    typedef T V4 __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    const int i = (int)blockIdx.x * (256 / L) + (int)threadIdx.x / L;
    const int n0 = ((int)threadIdx.x % L) * 4;
    const bool real = i < a.channels;
    const int ch = real ? i : a.channels - 1;
    const int s = (int)blockIdx.y;
    int lo, hi;
    seq_range(a.q, s, &lo, &hi);
    if (lo >= hi) return;
    const int grp = a.groups == 1 ? 0 : ch / a.per;
    const int left = min(4, a.dstate - n0);       // states of the lane that exist, none or fewer for the last lanes
    float h[4], rate[4];
    float* kept = a.state ? a.state + ((int64_t)s * a.channels + ch) * a.dstate + n0 : nullptr;
    if (kept) ss_load<4>(kept, left, h);
    else {
#pragma unroll
        for (int k = 0; k < 4; ++k) h[k] = 0.0f;
    }
    ss_load<4>(a.a + (int64_t)ch * a.dstate + n0, left, rate);
    const float bias = a.dt_bias ? a.dt_bias[ch] : 0.0f;
    const float dv = a.d ? a.d[ch] : 0.0f;
    for (int t = lo; t < hi; ++t) {
        const float x = (float)((const T*)a.x)[(int64_t)t * a.x_stride + ch];
        float step = (float)((const T*)a.dt)[(int64_t)t * a.dt_stride + ch] + bias;
        const float z = a.z ? (float)((const T*)a.z)[(int64_t)t * a.z_stride + ch] : 0.0f;
        const T* bp = (const T*)a.b + (int64_t)t * a.b_stride + (int64_t)grp * a.dstate + n0;
        const T* cp = (const T*)a.c + (int64_t)t * a.c_stride + (int64_t)grp * a.dstate + n0;
        float bv[4], cv[4];
        if (left == 4) {
            const V4 b4 = *(const V4*)bp, c4 = *(const V4*)cp;
#pragma unroll
            for (int k = 0; k < 4; ++k) { bv[k] = (float)b4[k]; cv[k] = (float)c4[k]; }
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                bv[k] = k < left ? (float)bp[k] : 0.0f;
                cv[k] = k < left ? (float)cp[k] : 0.0f;
            }
        }
        if (a.softplus) step = ss_softplus(step);
        const float in = step * x;
        step = ss_base2(step);
        float y = 0.0f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            h[k] = k < left ? fmaf(bv[k], in, ss_exp2(step * rate[k]) * h[k]) : 0.0f;
            y = fmaf(cv[k], h[k], y);
        }
        y = ss_sum<L>(y);
        y = fmaf(dv, x, y);
        if (a.z) y *= ss_silu<T>(z);
        if (n0 == 0 && real) ((T*)a.y)[(int64_t)t * a.y_stride + ch] = (T)y;
    }
    if (real && kept) ss_store<4>(kept, left, h);
}

template <typename T, int NS, int L, int PASS, bool FULL>
hipError_t launch_scan_pass(const SsArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)(PASS == SCAN_WHOLE ? a.q.seqs : a.slots), (unsigned)(a.groups * a.blocks_per_group));
    CADNN_LAUNCH((scan_kernel<T, NS, L, PASS, FULL>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

// How a call is worked on, from its sizes alone.
struct ScanPlan {
    int few;                  // few tokens a sequence
    int ns, lanes;            // states of a lane, lanes of a channel
    int blocks_per_group;
    int chunk;                // tokens of a piece; 0: whole sequences
    int longest;              // tokens of the longest sequence, as far as is known
    int64_t slots;
    size_t part_bytes, bytes;
};

ScanPlan plan_scan(const cadnn_scan_args& g) {
    ScanPlan p{};
    const int per = g.channels / g.groups;
    p.ns = g.dstate <= 8 ? 8 : 16;
    p.lanes = 1;
    while (p.ns * p.lanes < g.dstate) p.lanes *= 2;
    const int ch = 256 / p.lanes;
    p.blocks_per_group = (per + ch - 1) / ch;
    // The longest sequence, which decides, is known where all have one length or the caller says; of ragged ones it may be any, and as
    // one long prompt among single tokens would take a pass over whole sequences twenty times what pieces take, a quarter of the tokens
    // is supposed to be one sequence where there are many.
    const int average = g.tokens / g.seqs;
    const int longest = !g.seq_start ? average : g.longest > 0 ? std::max(g.longest, average) : g.tokens < 512 ? average : std::max(average, g.tokens / 4);
    p.longest = longest;
    // (64 sequences x 2048 channels x 16 states, fp16: 1 token 5.8 us here and 8.9 by the kernel for long sequences, 2 tokens 7.1, 9.1, 4 tokens 9.9, 9.7)
    p.few = longest <= 4;
    if (p.few) return p;
    // A wave alone on its SIMD takes 0.36 us a token and 3.5 more, whatever there is beside it on the chip; full, the chip takes 0.5 us for
    // a token of 1024 waves, both passes over pieces and their join together, which cost 12 us more to begin with.  (2048 channels x 16, us whole
    // and in pieces: one sequence of 64 tokens 26.8, 20.5, of 1024 tokens 371, 37; 4 of 64 tokens 27.2, 23.0; 16 of 256 tokens 98, 81; 16 of 64 tokens
    // of 512 channels 27.2, 22.6; 16 x 1024 channels x 64 states, 1024 tokens 413 and by these figures 524.)
    // Pieces are the longest that make 2560 waves, for up to four of a SIMD; more of them cost the join what they give the passes (us at 4096 x 2048 x 16,
    // fp16, passes and join: pieces of 64 tokens 35.5 + 44.9 + 6.6, of 32 tokens 32.7 + 41.0 + 11.4; 1501 x 1000 x 64, fp32, 9 sequences: 64 tokens 32.0 + 39.1 +
    // 7.3, 32 tokens 28.9 + 33.8 + 9.3, 16 tokens 27.3 + 31.5 + 35).
    const int64_t blocks = (int64_t)g.groups * p.blocks_per_group;
    p.chunk = 512;
    while (p.chunk > 16 && seq_slots(g.tokens, g.seqs, g.seq_start != nullptr, p.chunk) * blocks * 4 < 2560) p.chunk /= 2;
    const double whole = (3.5 + 0.36 * longest) * (double)((g.seqs * blocks * 4 + 1023) / 1024);
    const double pieces = 12.0 + std::max(0.5 * (double)g.tokens * (double)(blocks * 4) / 1024.0, 0.72 * p.chunk);
    if (whole <= pieces) {
        p.chunk = 0;
        return p;
    }
    p.slots = seq_slots(g.tokens, g.seqs, g.seq_start != nullptr, p.chunk);
    p.part_bytes = (size_t)p.slots * g.channels * g.dstate * 4;
    p.bytes = p.part_bytes + (size_t)p.slots * g.channels * 4;
    return p;
}

template <typename T, int NS, int L, bool FULL>
hipError_t launch_scan_passes(const SsArgs& a, hipStream_t s) {
    if (!a.part) return launch_scan_pass<T, NS, L, SCAN_WHOLE, FULL>(a, s);
    hipError_t e = launch_scan_pass<T, NS, L, SCAN_ENDS, FULL>(a, s);
    if (e != hipSuccess) return e;
    const int64_t per_seq = (int64_t)a.channels * a.dstate;
    if (a.longest > 16 * a.chunk) CADNN_LAUNCH(scan_join_kernel, dim3((unsigned)((per_seq + 63) / 64), (unsigned)a.q.seqs), dim3(256), 0, s, a);
    else CADNN_LAUNCH(scan_join_few_kernel, dim3((unsigned)((per_seq + 255) / 256), (unsigned)a.q.seqs), dim3(256), 0, s, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    return launch_scan_pass<T, NS, L, SCAN_PIECES, FULL>(a, s);
}

template <typename T, int NS, int L>
hipError_t launch_scan_lanes(const SsArgs& a, hipStream_t s) {
    return a.dstate == NS * L ? launch_scan_passes<T, NS, L, true>(a, s) : launch_scan_passes<T, NS, L, false>(a, s);
}

template <typename T, int L>
hipError_t launch_few_lanes(const SsArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)((a.channels + 256 / L - 1) / (256 / L)), (unsigned)a.q.seqs);
    CADNN_LAUNCH((scan_few_kernel<T, L>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_scan(const SsArgs& a, const ScanPlan& p, hipStream_t s) {
    if (p.few) {
        const int n = a.dstate;
        return n <= 4 ? launch_few_lanes<T, 1>(a, s) : n <= 8 ? launch_few_lanes<T, 2>(a, s) : n <= 16 ? launch_few_lanes<T, 4>(a, s)
             : n <= 32 ? launch_few_lanes<T, 8>(a, s) : n <= 64 ? launch_few_lanes<T, 16>(a, s) : n <= 128 ? launch_few_lanes<T, 32>(a, s)
             : launch_few_lanes<T, 64>(a, s);
    }
    if (p.ns == 8) return launch_scan_lanes<T, 8, 1>(a, s);
    switch (p.lanes) {
        case 1: return launch_scan_lanes<T, 16, 1>(a, s);
        case 2: return launch_scan_lanes<T, 16, 2>(a, s);
        case 4: return launch_scan_lanes<T, 16, 4>(a, s);
        case 8: return launch_scan_lanes<T, 16, 8>(a, s);
        default: return launch_scan_lanes<T, 16, 16>(a, s);
    }
}

cadnn_status check_scan(const char* who, const cadnn_scan_args* g) {
    if (!g) return fail(CADNN_EINVAL, "%s: NULL arguments", who);
    if (g->dtype != CADNN_F32 && g->dtype != CADNN_F16) return fail(CADNN_EINVAL, "%s: unknown dtype %d", who, (int)g->dtype);
    cadnn_status st = check_sequences(who, g->tokens, g->seqs, g->seq_start);
    if (st != CADNN_OK) return st;
    if (g->channels <= 0 || g->dstate <= 0 || g->groups <= 0 || g->longest < 0) return fail(CADNN_EINVAL, "%s: non-positive size", who);
    if (g->channels % g->groups) return fail(CADNN_EINVAL, "%s: %d channels in %d groups", who, g->channels, g->groups);
    if (g->dstate > kScanMaxStates) return fail(CADNN_EUNSUPPORTED, "%s: %d states a channel (at most %d are served)", who, g->dstate, kScanMaxStates);
    if (g->channels > (1 << 20) || g->groups > 4096 || g->seqs > 65535) return fail(CADNN_EUNSUPPORTED, "%s: more than 2^20 channels, 4096 groups or 65535 sequences", who);
    if ((int64_t)g->groups * plan_scan(*g).blocks_per_group > 65535) return fail(CADNN_EUNSUPPORTED, "%s: too many channels for one launch", who);
    return CADNN_OK;
}

}  // namespace

}  // namespace cadnn

using namespace cadnn;

extern "C" cadnn_status cadnn_selective_scan_workspace_bytes(const cadnn_scan_args* args, size_t* bytes) {
    if (!bytes) return fail(CADNN_EINVAL, "cadnn_selective_scan_workspace_bytes: NULL pointer");
    *bytes = 0;
    cadnn_status st = check_scan("cadnn_selective_scan_workspace_bytes", args);
    if (st != CADNN_OK) return st;
    if (args->tokens > 0) *bytes = plan_scan(*args).bytes;
    return CADNN_OK;
}

extern "C" cadnn_status cadnn_selective_scan(const cadnn_scan_args* args, void* workspace, size_t workspace_bytes, void* stream) {
    const char* who = "cadnn_selective_scan";
    cadnn_status st = check_scan(who, args);
    if (st != CADNN_OK) return st;
    const cadnn_scan_args& g = *args;
    if (g.tokens == 0) return CADNN_OK;
    if (!g.x || !g.dt || !g.a || !g.b || !g.c || !g.y) return fail(CADNN_EINVAL, "%s: NULL tensor", who);
    if (g.y == g.x || g.y == g.dt || g.y == g.b || g.y == g.c || g.y == g.z || g.y == (const void*)g.state)
        return fail(CADNN_EINVAL, "%s: y must not overlap what is read", who);
    if (g.x_stride < g.channels || g.dt_stride < g.channels || g.y_stride < g.channels || (g.z && g.z_stride < g.channels))
        return fail(CADNN_EINVAL, "%s: rows overlap (a stride below the number of channels)", who);
    if (g.b_stride < (int64_t)g.groups * g.dstate || g.c_stride < (int64_t)g.groups * g.dstate)
        return fail(CADNN_EINVAL, "%s: rows overlap (a stride of b or c below groups * dstate)", who);
    const uintptr_t e = g.dtype == CADNN_F16 ? 2 : 4;
    if (((uintptr_t)g.x | (uintptr_t)g.dt | (uintptr_t)g.b | (uintptr_t)g.c | (uintptr_t)g.z | (uintptr_t)g.y) % e ||
        ((uintptr_t)g.a | (uintptr_t)g.d | (uintptr_t)g.dt_bias | (uintptr_t)g.state | (uintptr_t)workspace) % 4)
        return fail(CADNN_EINVAL, "%s: a misaligned pointer", who);
    const ScanPlan p = plan_scan(g);
    SsArgs a{};
    a.x = g.x; a.dt = g.dt; a.b = g.b; a.c = g.c; a.z = g.z; a.y = g.y;
    a.x_stride = g.x_stride; a.dt_stride = g.dt_stride; a.b_stride = g.b_stride; a.c_stride = g.c_stride; a.z_stride = g.z_stride; a.y_stride = g.y_stride;
    a.a = g.a; a.d = g.d; a.dt_bias = g.dt_bias; a.state = g.state;
    a.q = Sequences{g.seq_start, g.tokens, g.seqs};
    a.channels = g.channels; a.dstate = g.dstate; a.groups = g.groups; a.per = g.channels / g.groups; a.softplus = g.softplus ? 1 : 0;
    a.blocks_per_group = p.blocks_per_group;
    if (p.chunk > 0 && workspace && workspace_bytes >= p.bytes) {
        a.chunk = p.chunk;
        a.longest = p.longest;
        a.slots = p.slots;
        a.part = (float*)workspace;
        a.span = (float*)((char*)workspace + p.part_bytes);
    }
    CADNN_HIP(g.dtype == CADNN_F16 ? launch_scan<_Float16>(a, p, (hipStream_t)stream) : launch_scan<float>(a, p, (hipStream_t)stream));
    return CADNN_OK;
}
