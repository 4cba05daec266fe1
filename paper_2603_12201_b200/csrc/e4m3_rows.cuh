// What the kernels that write e4m3 rows share: eight values a 128-bit load, and their codes for a row's scale
//     scale = max(max |x|, 1e-12) / 448,   code = e4m3(x / scale)   round to nearest even, saturating.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <stdint.h>

namespace idxc {

constexpr float kE4m3Max = 448.0f;

struct Vec8 {            // 8 bf16 values as loaded by one 128-bit load
    uint4 raw;
    __device__ __forceinline__ float get(int i) const {
        const uint32_t w = i < 2 ? raw.x : (i < 4 ? raw.y : (i < 6 ? raw.z : raw.w));
        return __uint_as_float((i & 1) ? (w & 0xFFFF0000u) : (w << 16));
    }
};

// x / scale, correctly rounded, from the correctly rounded reciprocal r of the row's scale: the product x * r is within
// two units of the quotient and one residual step (both FMAs exact in their product) lands on the nearest float. Checked
// against the IEEE division for EVERY pair of a bf16 maximum and a bf16 value not above it, both signs: the e4m3 codes
// agree everywhere (the floats differ only where x is so small that the residual underflows, all of which are code 0).
// Written with the residual's sign flipped so that a zero keeps its sign. A division costs about three times as many
// instructions, and with eight of them per 128-bit load the kernel was bound by its instruction issue, not by HBM.
__device__ __forceinline__ float div_by_scale(float x, float scale, float r) {
    const float q = x * r;
    const float e = __fmaf_rn(q, scale, -x);
    return __fmaf_rn(-e, r, q);
}

template <bool EXACT_DIV>
__device__ __forceinline__ uint2 quantize8_impl(const Vec8& v, float scale, float r) {
    uint32_t lo = 0, hi = 0;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const float x0 = v.get(2 * p), x1 = v.get(2 * p + 1);
        const float2 y = EXACT_DIV ? make_float2(__fdiv_rn(x0, scale), __fdiv_rn(x1, scale))
                                   : make_float2(div_by_scale(x0, scale, r), div_by_scale(x1, scale, r));
        const uint32_t two = __nv_cvt_float2_to_fp8x2(y, __NV_SATFINITE, __NV_E4M3);   // .x in the low byte
        if (p < 2) lo |= two << (16 * p);
        else hi |= two << (16 * (p - 2));
    }
    return make_uint2(lo, hi);
}

__device__ __forceinline__ uint2 quantize8(const Vec8& v, float scale) {
    if (scale <= 3.0e38f) return quantize8_impl<false>(v, scale, __frcp_rn(scale));
    return quantize8_impl<true>(v, scale, 0.f);        // an infinite maximum: plain divisions (x / inf = 0)
}

}  // namespace idxc
