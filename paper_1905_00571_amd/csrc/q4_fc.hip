// Fully connected layer with 4-bit weights and one scale per group of inputs:
//
//   y[t][o] = act( sum_g s[o][g] * sum_{i in g} q[o][i] * x[t][i] + bias[o] ),   q in -8 .. 7
//
// The codes reach the matrix instructions as what they are, small integers, exact in fp16 and bf16; a group's sum is
// taken in fp32 and multiplied by its scale there, so that no weight is ever rounded.  fp32 activations are cut into three
// bf16 parts that add up to them exactly (8 bits each of 24), one matrix instruction per part.
#include <atomic>

#include "q4.h"

namespace cadnn {

namespace {

typedef _Float16 q4_h8 __attribute__((ext_vector_type(8)));
typedef _Float16 q4_h4 __attribute__((ext_vector_type(4)));
typedef _Float16 q4_h2 __attribute__((ext_vector_type(2)));
typedef __bf16 q4_b8 __attribute__((ext_vector_type(8)));
typedef float q4_f4 __attribute__((ext_vector_type(4)));
typedef uint32_t q4_u4 __attribute__((ext_vector_type(4)));

struct Q4Args {
    const uint32_t* codes;
    const void* scales;
    const void* x;
    void* y;
    const float* bias;
    int64_t x_stride, y_stride;
    int n, cin, cout, blocks, act;
};

// Eight codes of one lane as the right operand of a matrix instruction (the left one are activations, so that a lane's four sums
// are four tokens of one filter, which has one scale).
template <typename T> struct Q4Frag;
template <> struct Q4Frag<_Float16> {
    static constexpr int kParts = 1;
    typedef q4_h8 V;
    // 0x6400 | u is 1024 + u in fp16 and 0x6400 | 16 u is 1024 + 16 u: a subtraction, or a multiplication by 1/16 and a
    // subtraction, both exact, leave u - 8.
    static __device__ __forceinline__ V codes(uint32_t w) {
        const q4_h2 m = {(_Float16)1032.0f, (_Float16)1032.0f}, s = {(_Float16)0.0625f, (_Float16)0.0625f}, k = {(_Float16)72.0f, (_Float16)72.0f};
        const uint32_t v = w >> 8;
        union { V v8; q4_h2 v2[4]; } r;
        r.v2[0] = __builtin_bit_cast(q4_h2, (w & 0x000f000fu) | 0x64006400u) - m;
        r.v2[1] = __builtin_elementwise_fma(__builtin_bit_cast(q4_h2, (w & 0x00f000f0u) | 0x64006400u), s, -k);
        r.v2[2] = __builtin_bit_cast(q4_h2, (v & 0x000f000fu) | 0x64006400u) - m;
        r.v2[3] = __builtin_elementwise_fma(__builtin_bit_cast(q4_h2, (v & 0x00f000f0u) | 0x64006400u), s, -k);
        return r.v8;
    }
    static __device__ __forceinline__ void parts(const _Float16 (&v)[8], V (&out)[1]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) out[0][e] = v[e];
    }
    static __device__ __forceinline__ q4_f4 mul(V codes, V x, q4_f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, codes, c, 0, 0, 0); }
};
template <> struct Q4Frag<float> {
    static constexpr int kParts = 3;
    typedef q4_b8 V;
    // (codes as sixteenths: what the conversion of a signed nibble gives; the scales on the device are 16 times theirs)
    static __device__ __forceinline__ V codes(uint32_t w) {
        w ^= 0x88888888u;
        const uint32_t v = w >> 4;
        union { V v8; uint32_t u[4]; } r;
        // (a byte of w or of w >> 4 is selected by the conversion itself, which looks at its low four bits)
        auto code = [&](int nibble) {
            return __float_as_uint(__builtin_amdgcn_cvt_off_f32_i4((int)__builtin_amdgcn_ubfe(nibble & 1 ? v : w, 4 * (nibble & ~1), 8)));
        };
#pragma unroll
        for (int t = 0; t < 4; ++t) r.u[t] = __builtin_amdgcn_perm(code(4 + t), code(t), 0x07060302u);
        return r.v8;
    }
    // The parts are cut off, not rounded, so that a large value's first part stays finite; what is left of an infinity
    // (no number) is replaced by a finite value that the infinity swallows.  A no-number that keeps its payload in its low bits, all of them
    // signalling, would be cut to an infinity: canonical, it is a quiet one, whose mark is among the high bits.  (3 tokens 25088 -> 4096, groups of 32,
    // 25.3 us so, 24.6 without; pairs compared, and made canonical behind a branch, 26.3.)
    static __device__ __forceinline__ void parts(const float (&v)[8], V (&out)[3]) {
        union { V v8; uint32_t u[4]; } p[3];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            float lo = __builtin_canonicalizef(v[2 * t]), hi = __builtin_canonicalizef(v[2 * t + 1]);
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                p[k].u[t] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
                lo -= __uint_as_float(p[k].u[t] << 16);
                hi -= __uint_as_float(p[k].u[t] & 0xffff0000u);
                if (k == 0) {
                    lo = __builtin_amdgcn_fmed3f(lo, -0x1p121f, 0x1p121f);
                    hi = __builtin_amdgcn_fmed3f(hi, -0x1p121f, 0x1p121f);
                }
            }
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) out[k] = p[k].v8;
    }
    static __device__ __forceinline__ q4_f4 mul(V codes, V x, q4_f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, codes, c, 0, 0, 0); }
};

// The scales of a lane's filter for the groups of a block, as they are stored.
template <typename T, int GP>
struct Q4Scales {
    typedef T V __attribute__((ext_vector_type(GP)));
    V v;
    __device__ __forceinline__ void load(const T* at) { v = *(const V*)at; }
    __device__ __forceinline__ float operator[](int g) const { return (float)v[g]; }
};

// Eight activations from input i0 on; what lies behind the row's end, or in no row, is zero.  (Rows need not start at
// multiples of 16 bytes: the loads are as wide for any alignment.)
template <typename T>
__device__ __forceinline__ void q4_load_x(const T* row, int i0, int cin, bool real, T (&v)[8]) {
    constexpr int N = 16 / (int)sizeof(T);
    typedef T V __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
    if (i0 + 8 <= cin) {
#pragma unroll
        for (int k = 0; k < 8; k += N) {
            V p = (V)(T)0.0f;
            if (real) p = *(const V*)(row + i0 + k);
#pragma unroll
            for (int e = 0; e < N; ++e) v[k + e] = p[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = real && i0 + e < cin ? row[i0 + e] : (T)0.0f;
    }
}

// The same where the row is known to reach that far.
template <typename T>
__device__ __forceinline__ void q4_load_whole(const T* at, T (&v)[8]) {
    constexpr int N = 16 / (int)sizeof(T);
    typedef T V __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
#pragma unroll
    for (int k = 0; k < 8; k += N) {
        const V p = *(const V*)(at + k);
#pragma unroll
        for (int e = 0; e < N; ++e) v[k + e] = p[e];
    }
}

// The end of a tile: four tokens of one filter.
template <typename T>
__device__ __forceinline__ void q4_store(const Q4Args& a, int token, int filter, q4_f4 v) {
    if (filter >= a.cout) return;
    if (a.bias) v += a.bias[filter];
    if (a.act == CADNN_ACT_RELU) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = apply_act(v[e], CADNN_ACT_RELU);
    } else if (a.act == CADNN_ACT_SILU) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = apply_act(v[e], CADNN_ACT_SILU);
    }
    T* out = (T*)a.y + (int64_t)token * a.y_stride + filter;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (token + e < a.n) out[e * a.y_stride] = (T)v[e];
}

// Few tokens: the weights are read once and bound the kernel.  A workgroup owns 16 * RT filters and 16 * NT tokens and its
// waves split the inputs, block by block in turn, so that even one tile of filters is read by eight waves; their sums meet
// in LDS and are added in the waves' order.
template <typename T, int GP, int RT, int NT>
__global__ __launch_bounds__(512) void q4_few_kernel(const Q4Args a) {
    typedef Q4Frag<T> F;
    extern __shared__ __attribute__((aligned(16))) char q4_smem[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int j = lane & 15, g = lane >> 4;
    const int tile0 = blockIdx.x * RT, tiles = (a.cout + 15) / 16;
    const int token0 = blockIdx.y * 16 * NT;
    q4_f4 acc[RT][NT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[r][t] = (q4_f4){0.0f, 0.0f, 0.0f, 0.0f};
    const T* rows[NT];
    bool real[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int token = token0 + 16 * t + j;
        real[t] = token < a.n;
        rows[t] = (const T*)a.x + (int64_t)(real[t] ? token : 0) * a.x_stride;
    }
    for (int b = wave; b < a.blocks; b += waves) {
        q4_u4 w[RT];
        Q4Scales<T, GP> sc[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int tile = min(tile0 + r, tiles - 1);
            w[r] = *(const q4_u4*)(a.codes + ((int64_t)tile * a.blocks + b) * 256 + lane * 4);
            sc[r].load((const T*)a.scales + (((int64_t)tile * a.blocks + b) * 16 + j) * GP);
        }
        typename F::V xf[NT][4][F::kParts];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                T v[8];
                q4_load_x<T>(rows[t], b * 128 + s * 32 + g * 8, a.cin, real[t], v);
                F::parts(v, xf[t][s]);
            }
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            q4_f4 sum[NT];
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const typename F::V c = F::codes(w[r][s]);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    if (s % (4 / GP) == 0) sum[t] = (q4_f4){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int p = F::kParts - 1; p >= 0; --p) sum[t] = F::mul(c, xf[t][s][p], sum[t]);
                    if ((s + 1) % (4 / GP) == 0) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[r][t][e] = fmaf(sc[r][s / (4 / GP)], sum[t][e], acc[r][t][e]);
                    }
                }
            }
        }
    }
    q4_f4* part = (q4_f4*)q4_smem;       // [wave][r][t][lane]
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) part[((wave * RT + r) * NT + t) * 64 + lane] = acc[r][t];
    __syncthreads();
    for (int i = wave; i < RT * NT; i += waves) {
        q4_f4 v = part[i * 64 + lane];
        for (int k = 1; k < waves; ++k) v += part[(k * RT * NT + i) * 64 + lane];
        q4_store<T>(a, token0 + 16 * (i % NT) + 4 * g, (tile0 + i / NT) * 16 + j, v);
    }
}

// As many tokens as one matrix instruction has columns: 16 in fp16, five in fp32, where the three parts of a token take three
// columns and one instruction serves all of them.  The workgroup brings the activations of a chunk (one block for every
// wave) into LDS, each element read, and cut apart, once, while the matrix instructions work on the chunk before, and a wave's
// codes and scales are fetched D chunks ahead.  us at 8192 -> 8192, groups of 128, one token: fp16 8.7, fp32 11.7, where the kernel above
// takes 14.1 and 19.0; the 35 MB are 6.4 us at the rate of a large copy.  (Fetched 3, 4, 8 chunks ahead, which repeats the last block as often behind the
// end: fp16 9.4, 9.8, 11.7; not fetched there, by a branch: 9.7, as what is waited for is then less well known.)
// (Two workgroups to a compute unit, which takes 128 registers: with one, the 257 tiles of 4099 filters took twice the time of 256.)
template <typename T, int GP, int HELD>
__global__ __launch_bounds__(512, 4) void q4_columns_kernel(const Q4Args a) {
    typedef Q4Frag<T> F;
    constexpr int P = F::kParts;
    constexpr int D = 2;

    extern __shared__ __attribute__((aligned(16))) char q4_smem[];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = (int)blockDim.x >> 6;
    const int j = lane & 15, g = lane >> 4;
    const int tile = (int)blockIdx.x;
    const uint32_t buf_bytes = (uint32_t)waves * 4096u;        // [block][16 columns][128 inputs], pieces of 16 bytes placed as below
    auto at = [&](uint32_t buf, int block, int col, int piece) { return q4_smem + buf * buf_bytes + block * 4096 + col * 256 + ((piece ^ col) << 4); };
    for (uint32_t i = (uint32_t)tid * 16u; i < 2 * buf_bytes; i += blockDim.x * 16u) *(q4_u4*)(q4_smem + i) = (q4_u4){0u, 0u, 0u, 0u};
    __syncthreads();
    const T* x = (const T*)a.x;
    const int per_token = 16 * waves;
    T held[HELD][8];                              // HELD pieces of a chunk are a thread's: a quarter of the tokens
    auto fetch = [&](int chunk) {
        const bool whole = (chunk + 1) * waves * 128 <= a.cin;       // (no row ends in the chunk: one wide load a piece)
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
            const int i = k * 64 * waves + tid, token = i / per_token, r = i - token * per_token;
            if (token < a.n) {
                const T* from = x + (int64_t)token * a.x_stride;
                if (whole) q4_load_whole<T>(from + chunk * waves * 128 + r * 8, held[k]);
                else q4_load_x<T>(from, chunk * waves * 128 + r * 8, a.cin, true, held[k]);
            }
        }
    };
    auto put = [&](uint32_t buf) {
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
            const int i = k * 64 * waves + tid, token = i / per_token, r = i - token * per_token;
            if (token < a.n) {
                typename F::V parts[P];
                F::parts(held[k], parts);
#pragma unroll
                for (int p = 0; p < P; ++p) *(typename F::V*)at(buf, r >> 4, token * P + p, r & 15) = parts[p];
            }
        }
    };
    q4_u4 w[D];
    Q4Scales<T, GP> sc[D];
    q4_f4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    const uint32_t* const code_at = a.codes + (int64_t)tile * a.blocks * 256 + lane * 4;
    const T* const scale_at = (const T*)a.scales + (int64_t)tile * a.blocks * (GP * 16) + j * GP;
    auto codes = [&](int slot, int chunk) {
        const int b = min(chunk * waves + wave, a.blocks - 1);      // (behind the last block the activations are zero)
        w[slot] = *(const q4_u4*)(code_at + (int64_t)b * 256);
        sc[slot].load(scale_at + (int64_t)b * (GP * 16));
    };
#pragma unroll
    for (int d = 0; d < D; ++d) codes(d, d);
    fetch(0);
    put(0);
    __syncthreads();
    const int chunks = (a.blocks + waves - 1) / waves;
    uint32_t buf = 0;
    for (int c0 = 0; c0 < chunks; c0 += D) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
            const int c = c0 + d;
            if (c < chunks) {
                if (c + 1 < chunks) fetch(c + 1);
                q4_f4 sum;
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const typename F::V xf = *(const typename F::V*)at(buf, wave, j, s * 4 + g);
                    sum = F::mul(F::codes(w[d][s]), xf, s % (4 / GP) == 0 ? (q4_f4){0.0f, 0.0f, 0.0f, 0.0f} : sum);
                    if ((s + 1) % (4 / GP) == 0) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[e] = fmaf(sc[d][s / (4 / GP)], sum[e], acc[e]);
                    }
                }
                codes(d, c + D);
                if (c + 1 < chunks) put(buf ^ 1);
                __syncthreads();
                buf ^= 1;
            }
        }
    }
    // column c of filter f is element c % 4 of lane c / 4 * 16 + f
    float* part = (float*)q4_smem;       // [wave][lane][4]
    *(q4_f4*)(part + (wave * 64 + lane) * 4) = acc;
    __syncthreads();
    for (int i = tid; i < 16 * a.n; i += (int)blockDim.x) {
        const int f = i & 15, token = i >> 4, filter = tile * 16 + f;
        if (filter >= a.cout) continue;
        float v = 0.0f;
        for (int k = 0; k < waves; ++k)
            for (int p = P - 1; p >= 0; --p) {
                const int c = token * P + p;
                v += part[(k * 64 + (c >> 2) * 16 + f) * 4 + (c & 3)];
            }
        ((T*)a.y)[(int64_t)token * a.y_stride + filter] = (T)apply_act(v + (a.bias ? a.bias[filter] : 0.0f), a.act);
    }
}

template <typename T, int GP, int HELD>
hipError_t launch_columns(const Q4Args& a, hipStream_t s) {
    const int waves = a.blocks >= 8 ? 8 : a.blocks;
    const size_t lds = (size_t)waves * 8192;
    const dim3 grid((unsigned)((a.cout + 15) / 16));
    CADNN_LAUNCH((q4_columns_kernel<T, GP, HELD>), grid, dim3(64u * waves), lds, s, a);
    return hipGetLastError();
}

template <typename T, int GP, int RT, int NT>
hipError_t launch_few(const Q4Args& a, hipStream_t s) {
    const int tiles = (a.cout + 15) / 16;
    const int waves = a.blocks >= 8 ? 8 : a.blocks;
    const dim3 grid((unsigned)((tiles + RT - 1) / RT), (unsigned)((a.n + 16 * NT - 1) / (16 * NT)));
    const size_t lds = (size_t)waves * RT * NT * 64 * sizeof(q4_f4);
    CADNN_LAUNCH((q4_few_kernel<T, GP, RT, NT>), grid, dim3(64u * waves), lds, s, a);
    return hipGetLastError();
}

// Many tokens: the matrix cores bound the kernel.  A workgroup owns 64 * RW filters and BN tokens; each of its four waves owns
// 16 * RW filters, whose codes it loads straight into the lanes that need them and expands in registers (no other wave needs
// them), and all BN tokens, whose activations are staged in LDS, 128 inputs at a time.  The 16-byte pieces of a token's row
// lie in LDS at their place exclusive-or the token's number, so that the sixteen lanes that read the same piece of sixteen
// tokens meet all banks.  KS steps of 32 inputs are expanded at a time; their sums start from zero in the first matrix
// instruction and are multiplied by the group's scale into the fp32 accumulators, which for groups of 32 is as much vector
// work as there is matrix work.  (With the scale multiplied into the codes, rounded to fp16, 2048 tokens through 4096 -> 8192 took 128 us for
// any group, where this takes 137 to 143, 147 to 151 and 168 to 173 for groups of 128, 64 and 32; the library's fp16 product takes 108 to 114.)  WK = 2: two
// times four waves take the blocks in turn and add up, where there are too few workgroups to wait for each other's loads.
// DIRECT (fp16): activations go straight to LDS, into the second of two buffers, else through registers.
template <typename T, int GP, int RW, int BN, int KS, int WK, bool DIRECT>
__global__ __launch_bounds__(256 * WK, 2) void q4_tile_kernel(const Q4Args a) {
    typedef Q4Frag<T> F;
    constexpr int P = F::kParts, CT = BN / 16, BUF = BN * 256 * P;         // bytes of a staged block
    constexpr int NBUF = DIRECT ? 2 : 1;
    constexpr int PER = 4 / GP < KS ? 4 / GP : KS;                          // steps that share a scale, in a phase
    extern __shared__ __attribute__((aligned(16))) char q4_smem[];
    const int tid = (int)threadIdx.x & 255, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wk = WK == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 8);
    char* smem = q4_smem + wk * (NBUF * BUF);
    const int j = lane & 15, g = lane >> 4;
    const int tiles = (a.cout + 15) / 16;
    const int tile0 = ((int)blockIdx.x * 4 + wave) * RW;
    const int token0 = (int)blockIdx.y * BN;
    const int rows_here = min(BN, a.n - token0);
    const T* x0 = (const T*)a.x + (int64_t)token0 * a.x_stride;
    // what a thread stages: pieces of 8 inputs (16 bytes in fp16) of the block's BN x 16
    constexpr int PIECES = BN * 16 / 256;
    auto lds_at = [&](int buf, int part, int row, int piece) {
        return (uint32_t)(buf * BUF + part * BN * 256 + row * 256 + ((piece ^ (row & 15)) << 4));
    };
    T held[DIRECT ? 1 : PIECES][8];
    auto fetch = [&](int b) {                 // into registers
        if constexpr (!DIRECT) {
            // (a row behind the last token repeats the first: its sums are not stored)
            const bool whole = (b + 1) * 128 <= a.cin;
#pragma unroll
            for (int k = 0; k < PIECES; ++k) {
                const int i = k * 256 + tid, row = i >> 4, at = b * 128 + (i & 15) * 8;
                const T* from = x0 + (int64_t)(row < rows_here ? row : 0) * a.x_stride;
                if (whole) q4_load_whole<T>(from + at, held[k]);
                else q4_load_x<T>(from, at, a.cin, true, held[k]);
            }
        }
    };
    auto put = [&](int buf) {                 // ... and from there to LDS
        if constexpr (!DIRECT) {
#pragma unroll
            for (int k = 0; k < PIECES; ++k) {
                const int i = k * 256 + tid, row = i >> 4, piece = i & 15;
                typename F::V parts[P];
                F::parts(held[k], parts);
#pragma unroll
                for (int p = 0; p < P; ++p) *(typename F::V*)(smem + lds_at(buf, p, row, piece)) = parts[p];
            }
        }
    };
    __amdgpu_buffer_rsrc_t rsrc;
    uint32_t voff[DIRECT ? PIECES : 1];
    if constexpr (DIRECT) {
        const uint32_t span = (uint32_t)((rows_here - 1) * a.x_stride + a.cin) * 2u;
        rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)x0, 0, span, 0x00020000);
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            const int i = k * 256 + tid, row = i >> 4, piece = (i & 15) ^ (row & 15);
            voff[k] = row < rows_here ? (uint32_t)(row * a.x_stride + piece * 8) * 2u : 0xffffffffu;
        }
    }
    auto copy = [&](int b, int buf) {         // straight to LDS: a wave's 64 pieces follow each other there, so the pieces are permuted as they are read
        if constexpr (DIRECT) {
#pragma unroll
            for (int k = 0; k < PIECES; ++k) {
                const int piece = (tid & 15) ^ (((k * 256 + tid) >> 4) & 15);
                const bool in = b * 128 + piece * 8 < a.cin && voff[k] != 0xffffffffu;
                const uint32_t off = in ? voff[k] + (uint32_t)b * 256u : 0xfffffff0u;       // (behind the buffer's end: zero)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)(smem + buf * BUF + (k * 256 + wave * 64) * 16),
                                                         16, off, 0, 0, 0);
            }
        }
    };
    q4_f4 acc[RW][CT];
#pragma unroll
    for (int r = 0; r < RW; ++r)
#pragma unroll
        for (int c = 0; c < CT; ++c) acc[r][c] = (q4_f4){0.0f, 0.0f, 0.0f, 0.0f};
    const uint32_t* code_at[RW];
    const T* scale_at[RW];
#pragma unroll
    for (int r = 0; r < RW; ++r) {
        const int tile = min(tile0 + r, tiles - 1);
        code_at[r] = a.codes + (int64_t)tile * a.blocks * 256 + lane * 4;
        scale_at[r] = (const T*)a.scales + (int64_t)tile * a.blocks * GP * 16 + j * GP;
    }
    const int steps = (a.blocks + WK - 1) / WK;
    q4_u4 w[RW];
#pragma unroll
    for (int r = 0; r < RW; ++r) w[r] = *(const q4_u4*)(code_at[r] + (int64_t)min(wk, a.blocks - 1) * 256);
    if constexpr (DIRECT) {
        copy(wk, 0);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    } else {
        fetch(wk);
        put(0);
    }
    __syncthreads();
    int buf = 0;
    for (int i = 0; i < steps; ++i) {
        const int b = i * WK + wk, next = min(b + WK, a.blocks - 1);
        const bool more = i + 1 < steps;
        if (more) {
            if constexpr (DIRECT) copy(b + WK, buf ^ 1);
            else fetch(b + WK);
        }
        q4_u4 wn[RW];
#pragma unroll
        for (int r = 0; r < RW; ++r) wn[r] = *(const q4_u4*)(code_at[r] + (int64_t)next * 256);
        if (WK == 1 || b < a.blocks) {
            Q4Scales<T, GP> scales[RW];
#pragma unroll
            for (int r = 0; r < RW; ++r) scales[r].load(scale_at[r] + (int64_t)b * (GP * 16));
#pragma unroll
            for (int ph = 0; ph < 4 / KS; ++ph) {
                float sc[RW][KS / PER];
                typename F::V af[RW][KS];
#pragma unroll
                for (int r = 0; r < RW; ++r) {
#pragma unroll
                    for (int q = 0; q < KS / PER; ++q) sc[r][q] = scales[r][(ph * KS + q * PER) * GP / 4];
#pragma unroll
                    for (int s = 0; s < KS; ++s) af[r][s] = F::codes(w[r][ph * KS + s]);
                }
#pragma unroll
                for (int c = 0; c < CT; ++c) {
                    typename F::V xf[KS][P];
#pragma unroll
                    for (int s = 0; s < KS; ++s)
#pragma unroll
                        for (int p = 0; p < P; ++p)
                            xf[s][p] = *(const typename F::V*)(smem + lds_at(buf, p, c * 16 + j, (ph * KS + s) * 4 + g));
                    q4_f4 sum[RW];
#pragma unroll
                    for (int s = 0; s < KS; ++s) {
#pragma unroll
                        for (int p = P - 1; p >= 0; --p)
#pragma unroll
                            for (int r = 0; r < RW; ++r)
                                sum[r] = F::mul(af[r][s], xf[s][p], p == P - 1 && s % PER == 0 ? (q4_f4){0.0f, 0.0f, 0.0f, 0.0f} : sum[r]);
                        if ((s + 1) % PER == 0) {
#pragma unroll
                            for (int r = 0; r < RW; ++r)
#pragma unroll
                                for (int e = 0; e < 4; ++e) acc[r][c][e] = fmaf(sc[r][s / PER], sum[r][e], acc[r][c][e]);
                        }
                    }
                }
            }
        }
#pragma unroll
        for (int r = 0; r < RW; ++r) w[r] = wn[r];
        // (what a wave copies has arrived before it meets the others)
        if constexpr (DIRECT) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if constexpr (DIRECT) buf ^= 1;
        else if (more) {
            put(0);
            __syncthreads();
        }
    }
    if constexpr (WK == 2) {
        q4_f4* part = (q4_f4*)q4_smem;
        if (wk == 1) {
#pragma unroll
            for (int r = 0; r < RW; ++r)
#pragma unroll
                for (int c = 0; c < CT; ++c) part[(r * CT + c) * 256 + tid] = acc[r][c];
        }
        __syncthreads();
        if (wk == 1) return;
#pragma unroll
        for (int r = 0; r < RW; ++r)
#pragma unroll
            for (int c = 0; c < CT; ++c) acc[r][c] += part[(r * CT + c) * 256 + tid];
    }
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int r = 0; r < RW; ++r) q4_store<T>(a, token0 + c * 16 + 4 * g, (tile0 + r) * 16 + j, acc[r][c]);
}

// More than 64 KiB of dynamic LDS have to be asked for, once for a kernel on a device.
struct LargeLds {
    std::atomic<bool> asked[64] = {};
    hipError_t ask(const void* kernel, int bytes) {
        int device = 0;
        hipError_t e = hipGetDevice(&device);
        if (e != hipSuccess || (device < 64 && asked[device].load(std::memory_order_acquire))) return e;
        e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e == hipSuccess && device < 64) asked[device].store(true, std::memory_order_release);
        return e;
    }
};

template <typename T, int GP, int RW, int BN, int KS, int WK, bool DIRECT>
hipError_t launch_tile(const Q4Args& a, hipStream_t s) {
    constexpr int staged = (DIRECT ? 2 : 1) * BN * 256 * Q4Frag<T>::kParts * WK, joined = WK == 2 ? 64 * RW * BN * 4 : 0;
    constexpr int lds = staged > joined ? staged : joined;
    if constexpr (lds > 64 * 1024) {
        static LargeLds large;
        const hipError_t e = large.ask((const void*)q4_tile_kernel<T, GP, RW, BN, KS, WK, DIRECT>, lds);
        if (e != hipSuccess) return e;
    }
    const dim3 grid((unsigned)((a.cout + 64 * RW - 1) / (64 * RW)), (unsigned)((a.n + BN - 1) / BN));
    CADNN_LAUNCH((q4_tile_kernel<T, GP, RW, BN, KS, WK, DIRECT>), grid, dim3(256 * WK), lds, s, a);
    return hipGetLastError();
}

// What a kernel takes, in us for rows of 4096 inputs, from the number of its workgroups: `one` while every compute unit has at
// most one, then `full` for every `fit` of them, the last ones included, which run `fit` at a time -- or, where their times were in
// proportion to their number (1024 to `full`), for as many as there are.
struct Q4Cost {
    double one, full;
    int fit;
    double of(int64_t workgroups) const {
        if (workgroups <= 256) return one;
        return fit >= 1024 ? std::max(one, full * (double)workgroups / fit) : full * (double)((workgroups + fit - 1) / fit);
    }
};

// The kernels, as (filters) x (tokens) of a workgroup; tiles with the activations straight to LDS where the call allows it, else through registers.
enum Q4Kernel {
    Q4_COLUMNS_FEW,         // 16 filters, 4 tokens
    Q4_COLUMNS,             // 16 filters, all that one matrix instruction holds: 16 tokens, in fp32 5
    Q4_FEW_16x16, Q4_FEW_32x16, Q4_FEW_64x16, Q4_FEW_64x32,
    Q4_TILE_SMALL,          // fp16 64 x 32, fp32 128 x 32
    Q4_TILE_MIDDLE,         // fp16 128 x 64, fp32 256 x 32
    Q4_TILE_LARGE,          // fp16 128 x 128 (through registers 128 x 64, one block at a time), fp32 256 x 64
    Q4_TILE_SMALL_REGISTERS, Q4_TILE_MIDDLE_REGISTERS, Q4_TILE_LARGE_REGISTERS
};

// Which kernel.  Large tiles read and expand less, but a workgroup alone on its compute unit waits out every latency, and one
// more than fit costs a round; so the kernels are compared by what they were measured to take (random data, 4096 -> 4096, 33 to 2048
// tokens; groups of 128, 64, 32).  fp16, 128 x 128 / 128 x 64 / 64 x 32 tiles / few tokens: 128 tokens 50, 22, 13.7, 15; 512 tokens 51,
// 25, 29, 52; 2048 tokens 76, 85, 115, more.  fp16 through registers, rows of 4095 inputs, groups of 128 and 32, 128 x 64 one block at a time / 128 x 64 / 64 x 32 /
// few tokens: 64 tokens 35, 31, 15.6, 18.2 and 46, 37, 17.6, 19.1; 300 tokens 38, 34, 39, 75 and 49, 40, 43, 79; 515 tokens 50, 61, 58, 122 and 62, 77, 63, 133;
// 2047 tokens of 8190 filters 190, 255, 330, 894 and 264, 311, 365, 954.  (Few tokens where every compute unit has at most one workgroup: with rows of 1001 inputs,
// 50 tokens of 1000 filters, 5.7 against the small tile's 6.0 and 6.4.)
// fp32, 256 x 64 / 256 x 32 / 128 x 32 / few tokens: 128 tokens 90, 51, 34, 22; 512 tokens 91, 54, 57, 81;
// 2048 tokens 198, 216, 218, more.
template <typename T, int GP>
Q4Kernel choose_q4(const Q4Args& a) {
    auto workgroups = [&](int filters, int tokens) { return (int64_t)((a.cout + filters - 1) / filters) * ((a.n + tokens - 1) / tokens); };
    if (a.n > 32) {
        constexpr int G = GP == 1 ? 0 : GP == 2 ? 1 : 2;
        if constexpr (sizeof(T) == 2) {
            // straight to LDS: whole pieces of eight, and 32-bit offsets from the first token of a tile on
            const bool direct = (uintptr_t)a.x % 16 == 0 && a.x_stride % 8 == 0 && a.cin % 8 == 0 && a.x_stride < (1 << 22);
            if (direct) {
                constexpr Q4Cost large[3] = {{52, 75, 512}, {52, 83, 512}, {70, 97, 512}}, middle[3] = {{24, 38, 512}, {25, 52, 512}, {36, 65, 512}};
                constexpr Q4Cost small[3] = {{14, 28, 1024}, {15, 30, 1024}, {18, 37, 1024}}, few[3] = {{11.5, 17, 512}, {12.5, 18.5, 512}, {14, 21, 512}};
                const double l = large[G].of(workgroups(128, 128)), m = middle[G].of(workgroups(128, 64)), sm = small[G].of(workgroups(64, 32));
                const double f = few[G].of(workgroups(64, 16));
                if (l <= m && l <= sm && l <= f) return Q4_TILE_LARGE;
                if (m <= sm && m <= f) return Q4_TILE_MIDDLE;
                if (sm <= f) return Q4_TILE_SMALL;
            } else if (workgroups(64, 16) > 256) {
                constexpr Q4Cost large[3] = {{38, 110, 1024}, {40, 113, 1024}, {50, 142, 1024}}, middle[3] = {{33.5, 67, 512}, {35, 71, 512}, {41, 82, 512}};
                constexpr Q4Cost small[3] = {{16.5, 54, 1024}, {17, 55, 1024}, {18.5, 59, 1024}};
                const double l = large[G].of(workgroups(128, 64)), m = middle[G].of(workgroups(128, 64)), sm = small[G].of(workgroups(64, 32));
                return l <= m && l <= sm ? Q4_TILE_LARGE_REGISTERS : m <= sm ? Q4_TILE_MIDDLE_REGISTERS : Q4_TILE_SMALL_REGISTERS;
            }
        } else {
            constexpr Q4Cost large[3] = {{93, 98, 256}, {96, 105, 256}, {106, 115, 256}}, middle[3] = {{52, 54, 256}, {54, 57, 256}, {59, 60, 256}};
            constexpr Q4Cost small[3] = {{38, 29, 256}, {39, 31, 256}, {41, 38, 256}}, few[3] = {{22.5, 20.5, 256}, {22.5, 20.5, 256}, {23, 21, 256}};
            constexpr Q4Cost fewer[3] = {{16.5, 25, 512}, {16.5, 29.5, 512}, {17, 29.5, 512}};
            const double l = large[G].of(workgroups(256, 64)), m = middle[G].of(workgroups(256, 32)), sm = small[G].of(workgroups(128, 32));
            const double f2 = few[G].of(workgroups(64, 32)), f1 = fewer[G].of(workgroups(64, 16)), f = std::min(f1, f2);
            if (l <= m && l <= sm && l <= f) return Q4_TILE_LARGE;
            if (m <= sm && m <= f) return Q4_TILE_MIDDLE;
            if (sm <= f) return Q4_TILE_SMALL;
            if (f2 <= f1 && workgroups(64, 32) >= 256) return Q4_FEW_64x32;
        }
    }
    // Staged activations pay from rows of some length on (one token, 512 -> 512: fp16 3.5 staged, 2.9 not; 4096 -> 4096: 4.3, 5.7).
    if (a.n <= 16 / Q4Frag<T>::kParts && a.blocks > (sizeof(T) == 2 ? 16 : 8)) return a.n <= 4 ? Q4_COLUMNS_FEW : Q4_COLUMNS;
    // (13 tokens, 5003 -> 4099, groups of 32, fp16: one tile of filters a wave 22.5, two 14.5; 4096 filters, one 13.5, two 14.5)
    if (a.n <= 16) return a.cout > 16 * 256 && a.blocks > 8 ? Q4_FEW_32x16 : Q4_FEW_16x16;
    constexpr bool h = sizeof(T) == 2;
    constexpr Q4Cost few1 = {h ? 7.3 : 11.3, h ? 12.5 : 20, 512}, few2 = {h ? 9.3 : 11.8, h ? 13 : 21.5, 512}, few4 = {h ? 11.5 : 16.5, h ? 16.5 : 27, 512};
    const double f1 = few1.of(workgroups(16, 16)), f2 = few2.of(workgroups(32, 16)), f4 = few4.of(workgroups(64, 16));
    return f4 <= f2 && f4 <= f1 ? Q4_FEW_64x16 : f2 <= f1 ? Q4_FEW_32x16 : Q4_FEW_16x16;
}

template <typename T, int GP>
hipError_t launch_q4(const Q4Args& a, hipStream_t s) {
    constexpr bool h = sizeof(T) == 2;
    const Q4Kernel kernel = choose_q4<T, GP>(a);
    switch (kernel) {
        case Q4_COLUMNS_FEW: return launch_columns<T, GP, 1>(a, s);
        case Q4_COLUMNS: return launch_columns<T, GP, h ? 4 : 2>(a, s);
        case Q4_FEW_16x16: return launch_few<T, GP, 1, 1>(a, s);
        case Q4_FEW_32x16: return launch_few<T, GP, 2, 1>(a, s);
        case Q4_FEW_64x16: return launch_few<T, GP, 4, 1>(a, s);
        default: break;
    }
    if constexpr (h) {
        switch (kernel) {
            case Q4_TILE_SMALL: return launch_tile<T, GP, 1, 32, 4, 2, true>(a, s);
            case Q4_TILE_MIDDLE: return launch_tile<T, GP, 2, 64, 4, 2, true>(a, s);
            case Q4_TILE_LARGE: return launch_tile<T, GP, 2, 128, GP == 1 ? 4 : 2, 1, true>(a, s);
            case Q4_TILE_SMALL_REGISTERS: return launch_tile<T, GP, 1, 32, 4, 2, false>(a, s);
            case Q4_TILE_MIDDLE_REGISTERS: return launch_tile<T, GP, 2, 64, 4, 2, false>(a, s);
            default: return launch_tile<T, GP, 2, 64, 4, 1, false>(a, s);
        }
    } else {
        switch (kernel) {
            case Q4_FEW_64x32: return launch_few<T, GP, 4, 2>(a, s);
            case Q4_TILE_SMALL: return launch_tile<T, GP, 2, 32, 4, 2, false>(a, s);
            case Q4_TILE_MIDDLE: return launch_tile<T, GP, 4, 32, 4, 2, false>(a, s);
            default: return launch_tile<T, GP, 4, 64, 2, 2, false>(a, s);
        }
    }
}

template <typename T>
hipError_t launch_q4_group(const Q4Args& a, int group, hipStream_t s) {
    return group == 128 ? launch_q4<T, 1>(a, s) : group == 64 ? launch_q4<T, 2>(a, s) : launch_q4<T, 4>(a, s);
}

template <typename T>
Q4Kernel choose_q4_group(const Q4Args& a, int group) {
    return group == 128 ? choose_q4<T, 1>(a) : group == 64 ? choose_q4<T, 2>(a) : choose_q4<T, 4>(a);
}

// A launch has at most 65535 rows of workgroups.
constexpr int kQ4LaunchRows = 16 * 65535;

// What choice and launch need of a call's first rows.
Q4Args q4_args(const cadnn_q4_weights* w, const void* x, int64_t x_stride, int n) {
    Q4Args a{};
    a.codes = (const uint32_t*)w->d_codes.p; a.scales = w->d_scales.p;
    a.x = x; a.x_stride = x_stride;
    a.n = std::min(kQ4LaunchRows, n); a.cin = w->cin; a.cout = w->cout; a.blocks = (w->cin + kQ4Block - 1) / kQ4Block;
    return a;
}

}  // namespace

const char* q4_fc_variant(const cadnn_q4_weights* w, const void* x, int64_t x_stride, int n) {
    const Q4Args a = q4_args(w, x, x_stride, n);
    const bool h = w->dtype == CADNN_F16;
    switch (h ? choose_q4_group<_Float16>(a, w->group) : choose_q4_group<float>(a, w->group)) {
        case Q4_COLUMNS_FEW: return "columns_4";
        case Q4_COLUMNS: return h ? "columns_16" : "columns_5";
        case Q4_FEW_16x16: return "few_16x16";
        case Q4_FEW_32x16: return "few_32x16";
        case Q4_FEW_64x16: return "few_64x16";
        case Q4_FEW_64x32: return "few_64x32";
        case Q4_TILE_SMALL: return h ? "tile_64x32_lds" : "tile_128x32";
        case Q4_TILE_MIDDLE: return h ? "tile_128x64_lds" : "tile_256x32";
        case Q4_TILE_LARGE: return h ? "tile_128x128_lds" : "tile_256x64";
        case Q4_TILE_SMALL_REGISTERS: return "tile_64x32";
        case Q4_TILE_MIDDLE_REGISTERS: return "tile_128x64";
        default: return "tile_128x64_whole";
    }
}

cadnn_status launch_q4_fc(const cadnn_q4_weights* w, const void* x, int64_t x_stride, void* y, int64_t y_stride, int n,
                          const float* bias, int act, hipStream_t s) {
    const size_t e = w->elem();
    for (int n0 = 0; n0 < n; n0 += kQ4LaunchRows) {
        Q4Args a = q4_args(w, (const char*)x + (size_t)n0 * x_stride * e, x_stride, n - n0);
        a.y = (char*)y + (size_t)n0 * y_stride * e; a.y_stride = y_stride;
        a.bias = bias; a.act = act;
        CADNN_HIP(w->dtype == CADNN_F16 ? launch_q4_group<_Float16>(a, w->group, s) : launch_q4_group<float>(a, w->group, s));
    }
    return CADNN_OK;
}

}  // namespace cadnn
