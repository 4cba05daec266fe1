// The two forms in which a latent cache row (512 value columns, 64 positional columns) is held, and how a row's bytes become
// bf16 operands. bf16: 1152 bytes, the columns in order. 4 bits: 416 bytes,
//   bytes   0..255  codes: a nibble u = code + 8 per value column; the word of columns 8g..8g+7 holds, from its lowest
//                   nibble up, columns 0 2 4 6 1 3 5 7 of the eight, so that (word >> 4i) & 0x000F000F is the pair (2i, 2i+1)
//   bytes 256..287  one bf16 scale per 32 columns, 5 significant bits
//   bytes 288..415  the positional columns in bf16
// A code has at most 4 significant bits (and only -8 has its own power of two), a scale 5: their product has at most 8, so
// code * scale is EXACT in bf16 and the reader's value is the stored value, with no second rounding.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

namespace idxc {

constexpr int kLatentCols = 576;
constexpr int kLatentValueCols = 512;
constexpr int kLatentBf16RowBytes = kLatentCols * 2;
constexpr int kLatentQ4RowBytes = 416;
constexpr int kLatentQ4ScaleOff = 256;
constexpr int kLatentQ4RopeOff = 288;

// Eight columns of a 4-bit row: `word` their codes, `scale2` the group's scale in both halves. 0x4300 | u is 128 + u in bf16
// (unit step 1 there), so the subtraction of 136 leaves the code exactly.
__device__ __forceinline__ uint4 dequant8_q4(uint32_t word, __nv_bfloat162 scale2) {
    uint32_t r[4];
    const uint32_t bias_bits = 0x43084308u;            // 136 in both halves
    const __nv_bfloat162 bias = *reinterpret_cast<const __nv_bfloat162*>(&bias_bits);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t t = ((word >> (4 * i)) & 0x000F000Fu) | 0x43004300u;
        const __nv_bfloat162 v = __hmul2(__hsub2(*reinterpret_cast<const __nv_bfloat162*>(&t), bias), scale2);
        r[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

__device__ __forceinline__ __nv_bfloat162 scale_pair(uint16_t bits) {
    const uint32_t two = static_cast<uint32_t>(bits) * 0x10001u;
    return *reinterpret_cast<const __nv_bfloat162*>(&two);
}

}  // namespace idxc
