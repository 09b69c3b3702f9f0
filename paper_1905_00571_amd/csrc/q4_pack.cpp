// Weights in 4 bits with one scale per group of inputs: quantisation, the canonical form on the host, the device layout
// and the entry points.
#include <cmath>
#include <cstring>
#include <new>

#include "q4.h"

namespace cadnn {

namespace {

cadnn_status check_q4(const char* who, int cout, int cin, int group, cadnn_dtype dtype) {
    if (cout <= 0 || cin <= 0) return fail(CADNN_EINVAL, "%s: non-positive size", who);
    if (dtype != CADNN_F32 && dtype != CADNN_F16) return fail(CADNN_EINVAL, "%s: unknown dtype %d", who, (int)dtype);
    if (group != 32 && group != 64 && group != 128) return fail(CADNN_EUNSUPPORTED, "%s: groups of %d inputs (32, 64 or 128 are served)", who, group);
    if (cin > (1 << 24) || cout > (1 << 24)) return fail(CADNN_EUNSUPPORTED, "%s: cin or cout above 2^24", who);
    return CADNN_OK;
}

// The scale as the storage type holds it.
inline float stored_scale(float s, cadnn_dtype dtype) { return dtype == CADNN_F16 ? f16_to_f32(f32_to_f16_rne(s)) : s; }

// (fp32 products are summed over codes / 16 and multiplied by 16 * scale, which has to be finite)
inline bool scale_ok(float s) { return std::isfinite(s) && std::fabs(s) < 0x1p120f; }

cadnn_status make_q4(int cout, int cin, int group, cadnn_dtype dtype, std::unique_ptr<cadnn_q4_weights>* out) {
    std::unique_ptr<cadnn_q4_weights> w(new cadnn_q4_weights());
    w->cout = cout; w->cin = cin; w->group = group; w->dtype = dtype;
    w->groups = (cin + group - 1) / group;
    w->codes.assign((size_t)cout * (((size_t)cin + 1) / 2), 0x88);
    w->scales.assign((size_t)cout * w->groups, 0.0f);
    *out = std::move(w);
    return CADNN_OK;
}

inline void put_code(uint8_t* row, int i, int code) {
    uint8_t& b = row[i >> 1];
    const int u = code + 8;
    b = i & 1 ? (uint8_t)((b & 0x0f) | u << 4) : (uint8_t)((b & 0xf0) | u);
}

inline int get_code(const uint8_t* row, int i) { return ((row[i >> 1] >> ((i & 1) * 4)) & 15) - 8; }

}  // namespace

// Device layout.  Filters come in tiles of 16, inputs in blocks of 128; a tile's blocks follow each other, 1024 bytes each:
// lane l of a wave owns the 16 bytes at 16 * l, filter l % 16 and, in dword s (a step of 32 inputs), the eight inputs
// 32 * s + 8 * (l / 16) onwards -- what one lane of a 16 x 16 x 32 matrix instruction holds of an operand, so that
// a wave reads whole kilobytes and moves nothing between lanes.  In a dword nibble t holds element 2t and nibble 4 + t
// element 2t + 1: a shift and a mask leave two neighbours in the two halves of the register.  Scales lie as
// [tile][block][16 filters][groups of the block]: one load for a lane, whose sums are all of one filter.  What lies behind the last filter or input has code 0 (8 as stored) and scale 0.
cadnn_status ensure_q4_device(const cadnn_q4_weights* w, const char* who, hipStream_t stream, bool has_stream) {
    std::lock_guard<std::mutex> lock(w->mu);
    int device = -1;
    CADNN_HIP(hipGetDevice(&device));
    if (w->device >= 0) {
        if (w->device != device) return fail(CADNN_EINVAL, "%s: the weights are on device %d, the current one is %d", who, w->device, device);
        return CADNN_OK;
    }
    if (has_stream) {
        hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
        CADNN_HIP(hipStreamIsCapturing(stream, &cap));
        if (cap != hipStreamCaptureStatusNone)
            return fail(CADNN_EINVAL, "%s: the first call uploads the weights and cannot be captured (cadnn_q4_prepare)", who);
    }
    const int tiles = (w->cout + kQ4Rows - 1) / kQ4Rows, blocks = (w->cin + kQ4Block - 1) / kQ4Block, per = kQ4Block / w->group;
    try {
        std::vector<uint32_t> words((size_t)tiles * blocks * 256, 0x88888888u);
        const size_t row_bytes = ((size_t)w->cin + 1) / 2;
        for (int o = 0; o < w->cout; ++o) {
            const uint8_t* row = w->codes.data() + (size_t)o * row_bytes;
            uint32_t* tile = words.data() + (size_t)(o / kQ4Rows) * blocks * 256 + (size_t)(o % kQ4Rows) * 4;
            for (int b = 0; b < blocks; ++b)
                for (int s = 0; s < 4; ++s)
                    for (int g = 0; g < 4; ++g) {
                        const int i0 = b * kQ4Block + s * 32 + g * 8;
                        uint32_t v = 0x88888888u;
                        if (i0 + 8 <= w->cin) {
                            // byte p holds elements 2p and 2p + 1, which go to nibbles p and 4 + p
                            uint32_t q;
                            std::memcpy(&q, row + i0 / 2, 4);
                            v = 0;
                            for (int p = 0; p < 4; ++p) v |= (q >> (8 * p) & 15u) << (4 * p) | (q >> (8 * p + 4) & 15u) << (16 + 4 * p);
                        } else {
                            for (int e = 0; e < 8 && i0 + e < w->cin; ++e) {
                                const int at = 4 * (e / 2) + 16 * (e & 1);
                                v = (v & ~(15u << at)) | (uint32_t)(get_code(row, i0 + e) + 8) << at;
                            }
                        }
                        tile[(size_t)b * 256 + g * 64 + s] = v;
                    }
        }
        cadnn_status st = w->d_codes.upload(words.data(), words.size() * 4);
        if (st != CADNN_OK) return st;
        const size_t padded = (size_t)tiles * blocks * per * kQ4Rows;
        std::vector<float> f;
        std::vector<uint16_t> h;
        if (w->dtype == CADNN_F16) h.assign(padded, 0);
        else f.assign(padded, 0.0f);
        for (int o = 0; o < w->cout; ++o)
            for (int g = 0; g < w->groups; ++g) {
                const size_t at = (((size_t)(o / kQ4Rows) * blocks + g / per) * kQ4Rows + o % kQ4Rows) * per + g % per;
                const float s = w->scales[(size_t)o * w->groups + g];
                if (w->dtype == CADNN_F16) h[at] = f32_to_f16_rne(s);
                else f[at] = 16.0f * s;      // (the kernels' fp32 codes are sixteenths)
            }
        st = w->dtype == CADNN_F16 ? w->d_scales.upload(h.data(), h.size() * 2) : w->d_scales.upload(f.data(), f.size() * 4);
        if (st != CADNN_OK) return st;
    } catch (const std::bad_alloc&) {
        return fail(CADNN_ENOMEM, "%s: out of host memory laying out 4-bit weights", who);
    }
    w->device = device;
    return CADNN_OK;
}

}  // namespace cadnn

using namespace cadnn;

extern "C" cadnn_status cadnn_q4_pack(const float* w_host, int cout, int cin, int group, cadnn_dtype dtype,
                                      cadnn_q4_weights** out) {
    if (out) *out = nullptr;
    if (!w_host || !out) return fail(CADNN_EINVAL, "cadnn_q4_pack: NULL pointer");
    cadnn_status st = check_q4("cadnn_q4_pack", cout, cin, group, dtype);
    if (st != CADNN_OK) return st;
    try {
        std::unique_ptr<cadnn_q4_weights> w;
        make_q4(cout, cin, group, dtype, &w);
        const size_t row_bytes = ((size_t)cin + 1) / 2;
        for (int o = 0; o < cout; ++o) {
            const float* src = w_host + (size_t)o * cin;
            uint8_t* row = w->codes.data() + (size_t)o * row_bytes;
            for (int g = 0; g < w->groups; ++g) {
                const int lo = g * group, hi = std::min(cin, lo + group);
                float top = 0.0f;
                bool finite = true;
                for (int i = lo; i < hi; ++i) {
                    top = std::max(top, std::fabs(src[i]));
                    finite = finite && std::isfinite(src[i]);
                }
                const float s = stored_scale(top / 7.0f, dtype);
                if (!finite || !scale_ok(s))
                    return fail(CADNN_EINVAL, "cadnn_q4_pack: row %d, inputs %d to %d: a weight that is not finite or too large for a scale", o, lo, hi - 1);
                w->scales[(size_t)o * w->groups + g] = s;
                for (int i = lo; i < hi; ++i) {
                    const float q = s > 0.0f ? std::nearbyint(src[i] / s) : 0.0f;
                    put_code(row, i, (int)std::min(7.0f, std::max(-8.0f, q)));
                }
            }
        }
        *out = w.release();
    } catch (const std::bad_alloc&) {
        return fail(CADNN_ENOMEM, "cadnn_q4_pack: out of host memory");
    }
    return CADNN_OK;
}

extern "C" cadnn_status cadnn_q4_pack_codes(const int8_t* codes_host, const float* scales_host, int cout, int cin, int group,
                                            cadnn_dtype dtype, cadnn_q4_weights** out) {
    if (out) *out = nullptr;
    if (!codes_host || !scales_host || !out) return fail(CADNN_EINVAL, "cadnn_q4_pack_codes: NULL pointer");
    cadnn_status st = check_q4("cadnn_q4_pack_codes", cout, cin, group, dtype);
    if (st != CADNN_OK) return st;
    try {
        std::unique_ptr<cadnn_q4_weights> w;
        make_q4(cout, cin, group, dtype, &w);
        for (size_t i = 0; i < w->scales.size(); ++i) {
            w->scales[i] = stored_scale(scales_host[i], dtype);
            if (!scale_ok(w->scales[i]))
                return fail(CADNN_EINVAL, "cadnn_q4_pack_codes: scale %zu is not finite or too large for its type", i);
        }
        const size_t row_bytes = ((size_t)cin + 1) / 2;
        for (int o = 0; o < cout; ++o) {
            const int8_t* src = codes_host + (size_t)o * cin;
            uint8_t* row = w->codes.data() + (size_t)o * row_bytes;
            uint8_t outside = 0;
            for (int i = 0; i + 1 < cin; i += 2) {
                const uint8_t a = (uint8_t)(src[i] + 8), b = (uint8_t)(src[i + 1] + 8);
                outside |= a | b;
                row[i / 2] = (uint8_t)(a | b << 4);
            }
            if (cin & 1) {
                const uint8_t a = (uint8_t)(src[cin - 1] + 8);
                outside |= a;
                row[cin / 2] = (uint8_t)(0x80 | a);
            }
            if (outside & 0xf0) return fail(CADNN_EINVAL, "cadnn_q4_pack_codes: row %d has a code outside -8..7", o);
        }
        *out = w.release();
    } catch (const std::bad_alloc&) {
        return fail(CADNN_ENOMEM, "cadnn_q4_pack_codes: out of host memory");
    }
    return CADNN_OK;
}

extern "C" cadnn_status cadnn_q4_free(cadnn_q4_weights* w) {
    delete w;
    return CADNN_OK;
}

extern "C" cadnn_status cadnn_q4_export(const cadnn_q4_weights* w, int8_t* codes, float* scales) {
    if (!w) return fail(CADNN_EINVAL, "cadnn_q4_export: NULL handle");
    const size_t row_bytes = ((size_t)w->cin + 1) / 2;
    if (codes)
        for (int o = 0; o < w->cout; ++o)
            for (int i = 0; i < w->cin; ++i)
                codes[(size_t)o * w->cin + i] = (int8_t)get_code(w->codes.data() + (size_t)o * row_bytes, i);
    if (scales) std::memcpy(scales, w->scales.data(), w->scales.size() * sizeof(float));
    return CADNN_OK;
}

extern "C" cadnn_status cadnn_q4_unpack(const cadnn_q4_weights* w, float* w_host_out) {
    if (!w || !w_host_out) return fail(CADNN_EINVAL, "cadnn_q4_unpack: NULL pointer");
    const size_t row_bytes = ((size_t)w->cin + 1) / 2;
    for (int o = 0; o < w->cout; ++o)
        for (int i = 0; i < w->cin; ++i)
            w_host_out[(size_t)o * w->cin + i] =
                w->scales[(size_t)o * w->groups + i / w->group] * (float)get_code(w->codes.data() + (size_t)o * row_bytes, i);
    return CADNN_OK;
}

extern "C" cadnn_status cadnn_q4_prepare(const cadnn_q4_weights* w) {
    if (!w) return fail(CADNN_EINVAL, "cadnn_q4_prepare: NULL handle");
    return ensure_q4_device(w, "cadnn_q4_prepare", nullptr, false);
}

extern "C" cadnn_status cadnn_q4_fc(const cadnn_q4_weights* w, const void* x, int64_t x_stride, void* y, int64_t y_stride, int n,
                                    const void* bias, int act, void* stream) {
    if (!w || !x || !y) return fail(CADNN_EINVAL, "cadnn_q4_fc: NULL pointer");
    if (n <= 0) return fail(CADNN_EINVAL, "cadnn_q4_fc: non-positive number of rows");
    if (x_stride < w->cin || y_stride < w->cout) return fail(CADNN_EINVAL, "cadnn_q4_fc: rows overlap (a stride below the row's length)");
    if (act != CADNN_ACT_NONE && act != CADNN_ACT_RELU && act != CADNN_ACT_SILU) return fail(CADNN_EINVAL, "cadnn_q4_fc: unknown activation %d", act);
    if (x == y) return fail(CADNN_EINVAL, "cadnn_q4_fc: y must not overlap x");
    if ((uintptr_t)x % w->elem() || (uintptr_t)y % w->elem() || (uintptr_t)bias % 4) return fail(CADNN_EINVAL, "cadnn_q4_fc: a misaligned pointer");
    if (n > (1 << 24)) return fail(CADNN_EUNSUPPORTED, "cadnn_q4_fc: more than 2^24 rows");
    cadnn_status st = ensure_q4_device(w, "cadnn_q4_fc", (hipStream_t)stream, true);
    if (st != CADNN_OK) return st;
    return launch_q4_fc(w, x, x_stride, y, y_stride, n, (const float*)bias, act, (hipStream_t)stream);
}

extern "C" cadnn_status cadnn_q4_fc_variant_name(const cadnn_q4_weights* w, const void* x, int64_t x_stride, int n, char* buf, size_t len) {
    if (!w || !buf || len == 0) return fail(CADNN_EINVAL, "cadnn_q4_fc_variant_name: NULL pointer");
    if (n <= 0 || x_stride < w->cin) return fail(CADNN_EINVAL, "cadnn_q4_fc_variant_name: non-positive number of rows, or rows that overlap");
    std::strncpy(buf, q4_fc_variant(w, x, x_stride, n), len - 1);
    buf[len - 1] = '\0';
    return CADNN_OK;
}
