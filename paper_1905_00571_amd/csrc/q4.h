// 4-bit weights with group scales: the handle and its launches.
#pragma once

#include "internal.h"

struct cadnn_q4_weights {
    int cout = 0, cin = 0, group = 0, groups = 0;
    cadnn_dtype dtype = CADNN_F32;
    // canonical form (host): code + 8 of weight (o, i) in nibble i & 1 of byte o * ((cin + 1) / 2) + i / 2,
    // scales[o * groups + g] as the storage type holds them
    std::vector<uint8_t> codes;
    std::vector<float> scales;
    // device layout (see q4_fc.hip), built by the first call or cadnn_q4_prepare
    mutable cadnn::DevBuf d_codes, d_scales;
    mutable int device = -1;
    mutable std::mutex mu;
    size_t elem() const { return dtype == CADNN_F16 ? 2 : 4; }
};

namespace cadnn {

constexpr int kQ4Rows = 16;       // filters of a tile of the device layout
constexpr int kQ4Block = 128;     // inputs of a tile; a group (32, 64 or 128) never straddles two

// y = act(x w^T + bias) on rows `x_stride` / `y_stride` elements apart; arguments are checked by the caller.
cadnn_status launch_q4_fc(const cadnn_q4_weights* w, const void* x, int64_t x_stride, void* y, int64_t y_stride, int n,
                          const float* bias, int act, hipStream_t s);
// Name of the kernel that serves the rows (the first 2^20 of them).
const char* q4_fc_variant(const cadnn_q4_weights* w, const void* x, int64_t x_stride, int n);
// Uploads the device layout, or checks that it is on the current device.  `capturing`: the call's stream, which must
// not be captured while memory is still to be allocated (NULL: none).
cadnn_status ensure_q4_device(const cadnn_q4_weights* w, const char* who, hipStream_t capturing, bool has_stream);

// v / (1 + exp(-v)), to about 6 half steps of the value (from -87 on; below, where exp(-v) passes what fp32 holds, to 1e-36): the exponent's
// product with log2(e) is taken in two parts, so that its rounding does not grow with v.  (Beyond 150 on either side, where the exponential is 0 or the
// quotient is, the parts could be infinite and their difference no number.)  A third of the instructions of the library's exponential and quotient,
// which bounded the fp16 convolution.
__device__ __forceinline__ float act_silu(float v) {
    const float u = __builtin_amdgcn_fmed3f(-v, -150.0f, 150.0f);
    const float hi = u * 1.44269502f, lo = fmaf(u, 1.44269502f, -hi) + u * 1.92596303e-8f;
    const float e = __builtin_amdgcn_exp2f(hi);
    return v * __builtin_amdgcn_rcpf(fmaf(e, fmaf(lo, 0.693147182f, 1.0f), 1.0f));
}

__device__ __forceinline__ float apply_act(float v, int act) {
    if (act == CADNN_ACT_RELU) return v > 0.0f ? v : 0.0f;
    if (act == CADNN_ACT_SILU) return act_silu(v);
    return v;
}

}  // namespace cadnn
