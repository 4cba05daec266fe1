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

// The first row of a sequence in an array of `rows` rows, brought into [-2^31, rows]: a position is below 2^31, so a base farther out names
// no row of the array either, and no sum of a base and a position wraps around.
__device__ __forceinline__ int64_t near_base(int64_t base, int64_t rows) {
    const int64_t low = -(int64_t(1) << 31);
    return base < low ? low : (base > rows ? rows : base);
}

// The scale of a group as the reader uses it, in both halves of a word: s and -24 s (3 s has at most 7 bits: exact).
struct Q4Scale {
    __nv_bfloat162 s, m24s;
};
__device__ __forceinline__ Q4Scale q4_scale_of(uint32_t bits) {      // the scale's bf16 bits in the low half
    const uint32_t two = __byte_perm(bits, 0u, 0x1010), c = 0xC1C0C1C0u;      // -24 in both halves
    Q4Scale r;
    r.s = *reinterpret_cast<const __nv_bfloat162*>(&two);
    r.m24s = __hmul2(r.s, *reinterpret_cast<const __nv_bfloat162*>(&c));
    return r;
}

// Eight columns of a 4-bit row: `word` their codes. A nibble in the upper four mantissa bits of 0x4180 is 16 + u = 24 + code, so
// (16 + u) s - 24 s = code * s with one FMA a pair, whose result is exact.
__device__ __forceinline__ uint4 dequant8_q4(uint32_t word, const Q4Scale& q) {
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t t = ((i == 0 ? word << 3 : word >> (4 * i - 3)) & 0x00780078u) | 0x41804180u;
        const __nv_bfloat162 v = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&t), q.s, q.m24s);
        r[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

// 32 bytes from a 32-byte aligned address, zeros if !use (nothing is read then).
__device__ __forceinline__ void load_nc_256(const uint8_t* at, bool use, uint32_t (&r)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = 0u;
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %9, 0;\n\t"
        "@p ld.global.nc.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\t}"
        : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7])
        : "l"(at), "r"(static_cast<uint32_t>(use)));
}

__device__ __forceinline__ uint32_t load_nc_32(const uint8_t* at, bool use) {
    uint32_t r = 0u;
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p ld.global.nc.b32 %0, [%1];\n\t}" : "+r"(r) : "l"(at), "r"(static_cast<uint32_t>(use)));
    return r;
}

}  // namespace idxc
