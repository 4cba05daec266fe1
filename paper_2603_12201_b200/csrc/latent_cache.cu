// Rows of a latent cache: written in 4 bits (with append), read back, and moved when a cache is compacted.
// The kernels are short and follow one another, so each may be launched while the one before it drains and waits for it at its top. Their
// inputs may be that one's outputs: they are read by plain loads (no __restrict__, no __ldg), which stay behind the wait.
#include "kernels.h"
#include "latent_format.cuh"
#include "ptx_sm100.cuh"

namespace idxc {
namespace {

constexpr int kRowsPerWarp = 2;          // rows whose loads a warp keeps in flight
constexpr int kRowThreads = 256;

__device__ __forceinline__ float bf16_at(const uint4& v, int i) {
    const uint32_t w = i < 2 ? v.x : (i < 4 ? v.y : (i < 6 ? v.z : v.w));
    return __uint_as_float((i & 1) ? (w & 0xFFFF0000u) : (w << 16));
}

constexpr float kScaleMax = 0x1.5p+123f;

// The smallest scale of 5 significant bits that holds `amax` in 7 steps: amax / 7 rounded up past its top 4 mantissa bits.
// At least 2^-100 (code * scale then stays far from the subnormals), at most 1.3125 * 2^123 (24 steps, which the reader
// subtracts, stay finite).
__device__ __forceinline__ float q4_scale(float amax) {
    const float s = __fdiv_rn(fmaxf(amax, 7.f * 0x1p-100f), 7.f);
    const float up = __uint_as_float((__float_as_uint(s) + 0x7FFFFu) & ~0x7FFFFu);
    return fminf(up, kScaleMax);
}

// One word of codes from eight columns, four instructions a column. x times the rounded reciprocal r of the scale is off by less than
// 2^-20, and an 8-bit number over a 5-bit one that is no half-integer is at least 2^-10 away from the next (below 7.5): so the sum with
// 6144, whose unit is 2^-11, rounds the quotient to a value on the same side of every border and puts exact halves exactly. The
// second sum rounds that to an integer, halves to even, in the low mantissa bits of 1.5 * 2^23 + 8 + code; the words' high
// parts, the same for every column, drop out of the weighted sum modulo 2^32 as one constant.
constexpr float kSnap = 6144.f;                          // 1.5 * 2^12
constexpr float kCodeBias = 12582912.f + 8.f;            // 1.5 * 2^23 + 8
constexpr uint32_t kWordBias = 0x4B400000u * 0x11111111u;
__device__ __forceinline__ uint32_t q4_word(const uint4& v, float r) {
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float y = __fadd_rn(__fmaf_rn(bf16_at(v, i), r, kSnap), kCodeBias - kSnap);
        word += __float_as_uint(y) << (4 * ((i & 1) * 4 + (i >> 1)));
    }
    return word - kWordBias;
}

// The same where codes may lie beyond +-7: the scale is at its upper limit, or x is not a number.
__device__ __noinline__ uint32_t q4_word_clipped(uint4 v, float scale) {
    uint32_t word = 0;
    for (int i = 0; i < 8; ++i) {
        const float y = rintf(__fdiv_rn(bf16_at(v, i), scale));
        word |= static_cast<uint32_t>(__float2int_rn(fminf(fmaxf(y, -7.f), 7.f)) + 8) << (4 * ((i & 1) * 4 + (i >> 1)));
    }
    return word;
}

// Largest magnitude of eight bf16 values, as bf16 bits; not a number if one is none (its group is then written clipped).
__device__ __forceinline__ uint32_t abs_max8(const uint4& v) {
    auto two = [](uint32_t w) -> __nv_bfloat162 {
        w &= 0x7FFF7FFFu;
        return *reinterpret_cast<const __nv_bfloat162*>(&w);
    };
    const __nv_bfloat162 m = __hmax2_nan(__hmax2_nan(two(v.x), two(v.y)), __hmax2_nan(two(v.z), two(v.w)));
    const uint32_t w = *reinterpret_cast<const uint32_t*>(&m);
    return max(w & 0xFFFFu, w >> 16);                    // (magnitudes: their bits are ordered as they are)
}

// A warp takes kRowsPerWarp rows; lane l holds the 8-column pieces l and l + 32 of a row's value columns, four lanes a group.
__global__ void __launch_bounds__(kRowThreads)
quantize_q4_kernel(const uint4* x, int64_t n, uint8_t* cache, int64_t cache_rows, const int64_t* dst_rows) {
    wait_for_previous();
    let_next_start();
    const int lane = threadIdx.x & 31;
    const int64_t row0 = (static_cast<int64_t>(blockIdx.x) * (kRowThreads / 32) + (threadIdx.x >> 5)) * kRowsPerWarp;
    uint4 v[kRowsPerWarp][2], rope[kRowsPerWarp];
    int64_t dst[kRowsPerWarp];
#pragma unroll
    for (int u = 0; u < kRowsPerWarp; ++u) {
        const bool in = row0 + u < n;
        const uint4* src = x + (row0 + u) * (kLatentCols / 8);
        v[u][0] = in ? src[lane] : make_uint4(0, 0, 0, 0);
        v[u][1] = in ? src[32 + lane] : make_uint4(0, 0, 0, 0);
        rope[u] = in && lane < 8 ? src[64 + lane] : make_uint4(0, 0, 0, 0);
        dst[u] = in ? (dst_rows ? dst_rows[row0 + u] : row0 + u) : -1;
    }
#pragma unroll
    for (int u = 0; u < kRowsPerWarp; ++u) {
        if (dst[u] < 0 || dst[u] >= cache_rows) continue;          // warp-uniform; a row outside the cache is not written
        uint8_t* out = cache + dst[u] * kLatentQ4RowBytes;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t m = abs_max8(v[u][h]);
            m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
            m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
            const float amax = __uint_as_float(m << 16);
            const float s = q4_scale(amax);
            reinterpret_cast<uint32_t*>(out)[h * 32 + lane] = amax <= 7.f * kScaleMax ? q4_word(v[u][h], __frcp_rn(s)) : q4_word_clipped(v[u][h], s);
            if ((lane & 3) == 0)
                reinterpret_cast<uint16_t*>(out + kLatentQ4ScaleOff)[h * 8 + (lane >> 2)] = static_cast<uint16_t>(__float_as_uint(s) >> 16);
        }
        if (lane < 8) reinterpret_cast<uint4*>(out + kLatentQ4RopeOff)[lane] = rope[u];
    }
}

// src_rows == nullptr: row r of the output is cache row r. A source row outside the cache gives zeros.
__global__ void __launch_bounds__(kRowThreads)
dequantize_q4_kernel(const uint8_t* cache, int64_t cache_rows, const int64_t* src_rows, int64_t n, uint4* out) {
    wait_for_previous();
    let_next_start();
    const int lane = threadIdx.x & 31;
    const int64_t row0 = (static_cast<int64_t>(blockIdx.x) * (kRowThreads / 32) + (threadIdx.x >> 5)) * kRowsPerWarp;
    uint32_t word[kRowsPerWarp][2];
    uint16_t scale[kRowsPerWarp][2];
    uint4 rope[kRowsPerWarp];
#pragma unroll
    for (int u = 0; u < kRowsPerWarp; ++u) {
        const int64_t src = row0 + u < n ? (src_rows ? src_rows[row0 + u] : row0 + u) : -1;
        const bool in = src >= 0 && src < cache_rows;
        const uint8_t* p = cache + (in ? src : 0) * kLatentQ4RowBytes;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            word[u][h] = in ? reinterpret_cast<const uint32_t*>(p)[h * 32 + lane] : 0x88888888u;
            scale[u][h] = in ? reinterpret_cast<const uint16_t*>(p + kLatentQ4ScaleOff)[h * 8 + (lane >> 2)] : static_cast<uint16_t>(0);
        }
        rope[u] = in && lane < 8 ? reinterpret_cast<const uint4*>(p + kLatentQ4RopeOff)[lane] : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < kRowsPerWarp; ++u) {
        if (row0 + u >= n) continue;
        uint4* dst = out + (row0 + u) * (kLatentCols / 8);
        dst[lane] = dequant8_q4(word[u][0], q4_scale_of(scale[u][0]));
        dst[32 + lane] = dequant8_q4(word[u][1], q4_scale_of(scale[u][1]));
        if (lane < 8) dst[64 + lane] = rope[u];
    }
}

// ---------------------------------------------------------------- compaction
// Row j of sequence b of the destination <- row keep[b][j] of sequence b of the source, j < n_keep[b], in units of T.
// Out of place the moves are independent: a block takes 1024 consecutive units of a sequence's rows, four a thread, whose four loads are in
// flight together. A row of the source is not read again, so it need not stay in the L2 (24 sequences of 900 to 6000 bf16 rows, choice and
// move: 28.4 -> 27.0 us).
constexpr int kCopyUnits = 1024;
template <typename T>
__global__ void __launch_bounds__(256)
compact_copy_kernel(const T* src, T* dst, uint32_t units, int64_t src_rows, int64_t dst_rows,
                    const int64_t* src_base, const int64_t* dst_base, const int32_t* keep, int ld_keep,
                    const int32_t* n_keep) {
    wait_for_previous();
    let_next_start();
    const int b = blockIdx.y;
    const int n = min(max(n_keep[b], 0), ld_keep);
    const int64_t sb = near_base(src_base[b], src_rows), db = near_base(dst_base[b], dst_rows);
    const int64_t total = static_cast<int64_t>(n) * units;
    const int32_t* k_row = keep + static_cast<int64_t>(b) * ld_keep;
    for (int64_t i0 = static_cast<int64_t>(blockIdx.x) * kCopyUnits; i0 < total; i0 += static_cast<int64_t>(gridDim.x) * kCopyUnits) {
        const int64_t j0 = i0 / units;                            // one long division a block
        const uint32_t u0 = static_cast<uint32_t>(i0 - j0 * units);
        int64_t from[4], to[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t o = u0 + k * 256 + threadIdx.x, dj = o / units, u = o - dj * units;
            const int64_t j = j0 + dj;
            from[k] = -1;
            if (j < n) {
                const int64_t p = k_row[j], s = sb + p, d = db + j;
                if (p >= 0 && s >= 0 && s < src_rows && d >= 0 && d < dst_rows) {
                    from[k] = s * units + u;
                    to[k] = d * units + u;
                }
            }
        }
        T v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (from[k] >= 0) v[k] = __ldcs(src + from[k]);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (from[k] >= 0) dst[to[k]] = v[k];
    }
}

// In place: keep is ascending, so keep[j] >= j, and a chunk of destination rows [a, b) overwrites no source of a later chunk
// (those are rows >= b). One CTA walks the chunks of one slice of a sequence's columns in order; within a chunk every load
// is done before the first store. Slices of columns are independent, which is where the parallelism comes from: four CTAs for a 4-bit row, one
// for a row of 128 bytes or less, and each chunk a round trip to memory. 8 sequences cut to 32768 rows: 4-bit rows 522 us, bf16 rows 544 us, sums
// 38 us; one of 128-byte keys 262 us. To another buffer the same take 42, 103, 3 and 3.5 us.
constexpr int kMoveThreads = 256;
constexpr int kMoveRowsPerThread = 8;
template <typename T>
__global__ void __launch_bounds__(kMoveThreads)
compact_in_place_kernel(T* rows, int units, int slice_units, int64_t n_rows, const int64_t* base,
                        const int32_t* keep, int ld_keep, const int32_t* n_keep) {
    wait_for_previous();
    let_next_start();
    const int b = blockIdx.y;
    const int n = min(max(n_keep[b], 0), ld_keep);
    const int64_t sb = near_base(base[b], n_rows);
    const int u0 = blockIdx.x * slice_units;
    const int width = min(slice_units, units - u0);
    const int per_pass = kMoveThreads / slice_units;          // rows that one pass of the CTA covers
    const int my_row = threadIdx.x / slice_units, my_unit = threadIdx.x % slice_units;
    const bool active = my_row < per_pass && my_unit < width;
    const int32_t* k_row = keep + static_cast<int64_t>(b) * ld_keep;
    for (int j0 = 0; j0 < n; j0 += per_pass * kMoveRowsPerThread) {
        T v[kMoveRowsPerThread];
        bool move[kMoveRowsPerThread];
#pragma unroll
        for (int i = 0; i < kMoveRowsPerThread; ++i) {
            const int j = j0 + i * per_pass + my_row;
            const int64_t k = active && j < n ? k_row[j] : -1;
            move[i] = k > j && sb + j >= 0 && sb + k < n_rows;       // keep[j] == j: the row is where it belongs
            if (move[i]) v[i] = rows[(sb + k) * units + u0 + my_unit];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kMoveRowsPerThread; ++i)
            if (move[i]) rows[(sb + j0 + i * per_pass + my_row) * units + u0 + my_unit] = v[i];
    }
}

}  // namespace

cudaError_t launch_quantize_q4(const void* x, int64_t n, void* cache, int64_t cache_rows, const int64_t* dst_rows, cudaStream_t stream) {
    const int64_t per_cta = kRowThreads / 32 * kRowsPerWarp;
    return launch_behind(quantize_q4_kernel, static_cast<unsigned>((n + per_cta - 1) / per_cta), kRowThreads, 0, stream,
                         static_cast<const uint4*>(x), n, static_cast<uint8_t*>(cache), cache_rows, dst_rows);
}

cudaError_t launch_dequantize_q4(const void* cache, int64_t cache_rows, const int64_t* src_rows, int64_t n, void* out, cudaStream_t stream) {
    const int64_t per_cta = kRowThreads / 32 * kRowsPerWarp;
    return launch_behind(dequantize_q4_kernel, static_cast<unsigned>((n + per_cta - 1) / per_cta), kRowThreads, 0, stream,
                         static_cast<const uint8_t*>(cache), cache_rows, src_rows, n, static_cast<uint4*>(out));
}

template <typename T>
static cudaError_t compact_as(const void* src, void* dst, int row_bytes, int64_t src_rows, int64_t dst_rows, const int64_t* src_base,
                              const int64_t* dst_base, const int32_t* keep, int ld_keep, const int32_t* n_keep, int B, cudaStream_t stream) {
    const int units = row_bytes / static_cast<int>(sizeof(T));
    if (src == dst) {
        const int slice = units < 8 ? units : 8;
        const dim3 grid(static_cast<unsigned>((units + slice - 1) / slice), static_cast<unsigned>(B));
        return launch_behind(compact_in_place_kernel<T>, grid, kMoveThreads, 0, stream, static_cast<T*>(dst), units, slice, dst_rows, src_base, keep, ld_keep, n_keep);
    }
    int64_t blocks = (static_cast<int64_t>(ld_keep) * units + kCopyUnits - 1) / kCopyUnits;
    const int64_t cap = 16 * 148 / B + 1;
    if (blocks > cap) blocks = cap;
    return launch_behind(compact_copy_kernel<T>, dim3(static_cast<unsigned>(blocks), static_cast<unsigned>(B)), 256, 0, stream, static_cast<const T*>(src),
                         static_cast<T*>(dst), static_cast<uint32_t>(units), src_rows, dst_rows, src_base, dst_base, keep, ld_keep, n_keep);
}

cudaError_t launch_compact_rows(const void* src, void* dst, int row_bytes, int64_t src_rows, int64_t dst_rows, const int64_t* src_base,
                                const int64_t* dst_base, const int32_t* keep, int ld_keep, const int32_t* n_keep, int B, cudaStream_t stream) {
    const uintptr_t both = reinterpret_cast<uintptr_t>(src) | reinterpret_cast<uintptr_t>(dst) | static_cast<uintptr_t>(row_bytes);
    if ((both & 15) == 0)
        return compact_as<uint4>(src, dst, row_bytes, src_rows, dst_rows, src_base, dst_base, keep, ld_keep, n_keep, B, stream);
    return compact_as<uint32_t>(src, dst, row_bytes, src_rows, dst_rows, src_base, dst_base, keep, ld_keep, n_keep, B, stream);
}

}  // namespace idxc
