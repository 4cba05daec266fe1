// The largest score that any key of a page could reach, from the page's bounds lo_d <= k_d <= hi_d:
//     u[b, g, p] = scale * max over the new tokens and heads of key head g of  sum_d max(q_d lo_d, q_d hi_d)
// With q = q+ + q- (its positive and its negative part) the sum is <q+, hi> + <q-, lo>: a matrix product over 2 d columns, q's rows against the
// pages' bounds as they lie in memory, in bf16 with fp32 accumulation (the parts of q are exact). Each bound is read once, 4 d bytes a page and
// head, for 4 d flops a query row: HBM-bound for the 1 to 64 rows of a decode step, so the products are warp-level MMAs that take the bounds
// straight from global memory as fragments. The columns are permuted alike in both operands so that a lane's share of four fragments is 16
// contiguous bytes; four lanes then read 64 contiguous bytes of a page, eight pages an instruction.
#include <cuda_bf16.h>

#include "kernels.h"
#include "ptx_sm100.cuh"

namespace idxc {
namespace {

constexpr int kWarps = 8;
constexpr int kMaxRows = 64;                     // query rows whose fragments fit in shared memory; more go in several rounds
constexpr float kForced = 3.0e38f;

struct ScoreArgsP {
    const __nv_bfloat16* bounds;
    int64_t n_pages;
    int P, H_kv;
    const __nv_bfloat16* q;
    int64_t q_stride;            // elements between the tokens of q
    int n_step, group;
    const int32_t* table;
    int64_t ld_table;
    const int32_t* lens;
    int keep_first, keep_last;
    float scale;
    float* scores;
    int64_t ld;
    int32_t* n_out;
    int groups_per_warp;         // of eight pages
    int heads;                   // key heads of a CTA: 1, 2, 4 or 8
};

// The positive or negative part of two elements of q. (volatile: formed where it is used. Held beside q for the whole loop, the parts push the bounds
// that are on their way out of the registers: 58 -> 86 us for 32 requests of 8K to 64K positions.)
template <bool POSITIVE>
__device__ __forceinline__ uint32_t part_of(uint32_t x) {
    uint32_t r;
    if (POSITIVE) asm volatile("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(0u));
    else asm volatile("min.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(0u));
    return r;
}

// FEW: at most 16 query rows; their fragments stay in registers.
template <int D, bool FEW>
__global__ void __launch_bounds__(kWarps * 32, 2)
page_scores_kernel(const ScoreArgsP a) {
    constexpr int KC = D / 32;                   // 64-byte pieces of a row of d columns
    __shared__ uint4 q_smem[FEW ? 1 : kMaxRows * D / 8];
    let_next_start();
    wait_for_previous();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, j = lane & 3;
    // The warps of a CTA take its heads of the same pages: a page's bounds lie side by side over the heads, and are read at about the same time.
    const int b = blockIdx.z, head = blockIdx.y * a.heads + warp % a.heads, slices = kWarps / a.heads;
    const int first = (blockIdx.x * a.groups_per_warp * slices + warp / a.heads) * 8, step = slices * 8;
    const int32_t* table = a.table + b * a.ld_table;
    auto page_of = [&](int p) -> int { return p < a.ld_table ? table[p] : -1; };
    int page_next = page_of(first + g);          // (on its way beside the length)
    const int64_t len = max(a.lens[b], 0);
    const int pages = static_cast<int>(min((len + a.P - 1) / a.P, a.ld_table));
    const int64_t out_row = static_cast<int64_t>(b) * a.H_kv + head;
    if (blockIdx.x == 0 && warp < a.heads && lane == 0) a.n_out[out_row] = pages;
    const int rows = a.n_step * a.group;
    if (static_cast<int>(blockIdx.x) * a.groups_per_warp * step >= pages) return;
    auto q_row = [&](int r) -> const uint4* {    // query row r: token r / group, head r % group of the key head's
        const int i = r / a.group;
        return reinterpret_cast<const uint4*>(a.q + (static_cast<int64_t>(b) * a.n_step + i) * a.q_stride +
                                              static_cast<int64_t>(head * a.group + (r - i * a.group)) * D);
    };
    const uint4 none = make_uint4(0u, 0u, 0u, 0u);
    uint4 qa[FEW ? KC : 1], qb[FEW ? KC : 1];    // rows g and g + 8
    if (FEW) {
#pragma unroll
        for (int c = 0; c < KC; ++c) {
            qa[FEW ? c : 0] = g < rows ? q_row(g)[4 * c + j] : none;
            qb[FEW ? c : 0] = g + 8 < rows ? q_row(g + 8)[4 * c + j] : none;
        }
    }
    for (int r0 = 0; r0 < rows; r0 += kMaxRows) {
        if (r0 > 0) page_next = page_of(first + g);
        const int n_rows = min(kMaxRows, rows - r0), tiles = FEW ? 1 : (n_rows + 15) / 16;
        if (!FEW) {
            __syncthreads();
            for (int i = threadIdx.x; i < tiles * 16 * (D / 8); i += kWarps * 32) {
                const int r = i / (D / 8), c = i - r * (D / 8);
                q_smem[FEW ? 0 : r * (D / 8) + (c ^ (r & 7))] = r < n_rows ? q_row(r0 + r)[c] : none;
            }
            __syncthreads();
        }
        // The bounds of the next eight pages are on their way while these are worked on.
        uint4 lo_next[KC], hi_next[KC];
        bool valid_next = false;
        auto fetch = [&](int p0) {
            const int64_t page = p0 + g < pages ? page_next : -1;
            valid_next = page >= 0 && page < a.n_pages;
            const uint4* edge = reinterpret_cast<const uint4*>(a.bounds) + ((valid_next ? page : 0) * a.H_kv + head) * (D / 4) + j;
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                lo_next[c] = valid_next ? edge[4 * c] : none;
                hi_next[c] = valid_next ? edge[D / 8 + 4 * c] : none;
            }
            page_next = page_of(p0 + step + g);
        };
        fetch(first);
        for (int i = 0, p0 = first; i < a.groups_per_warp && p0 < pages; ++i, p0 += step) {
            const bool valid = valid_next;
            uint4 lo[KC], hi[KC];
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                lo[c] = lo_next[c];
                hi[c] = hi_next[c];
            }
            if (i + 1 < a.groups_per_warp) fetch(p0 + step);
            float best0 = -INFINITY, best1 = -INFINITY;          // pages p0 + 2 j, + 1
            for (int t = 0; t < tiles; ++t) {
                float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < KC; ++c) {
                    uint4 x, y;
                    if (FEW) {
                        x = qa[FEW ? c : 0];
                        y = qb[FEW ? c : 0];
                    } else {
                        const int r = t * 16 + g;
                        x = q_smem[FEW ? 0 : r * (D / 8) + ((4 * c + j) ^ (r & 7))];
                        y = q_smem[FEW ? 0 : (r + 8) * (D / 8) + ((4 * c + j) ^ (r & 7))];
                    }
                    const uint32_t l0[4] = {part_of<false>(x.x), part_of<false>(y.x), part_of<false>(x.y), part_of<false>(y.y)};
                    const uint32_t l1[4] = {part_of<false>(x.z), part_of<false>(y.z), part_of<false>(x.w), part_of<false>(y.w)};
                    const uint32_t h0[4] = {part_of<true>(x.x), part_of<true>(y.x), part_of<true>(x.y), part_of<true>(y.y)};
                    const uint32_t h1[4] = {part_of<true>(x.z), part_of<true>(y.z), part_of<true>(x.w), part_of<true>(y.w)};
                    mma_16816<false>(acc, l0, lo[c].x, lo[c].y);
                    mma_16816<false>(acc, l1, lo[c].z, lo[c].w);
                    mma_16816<false>(acc, h0, hi[c].x, hi[c].y);
                    mma_16816<false>(acc, h1, hi[c].z, hi[c].w);
                }
                const int r = t * 16 + g;
                if (r < n_rows) {
                    best0 = fmaxf(best0, acc[0]);
                    best1 = fmaxf(best1, acc[1]);
                }
                if (r + 8 < n_rows) {
                    best0 = fmaxf(best0, acc[2]);
                    best1 = fmaxf(best1, acc[3]);
                }
            }
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) {
                best0 = fmaxf(best0, __shfl_xor_sync(0xFFFFFFFFu, best0, o));
                best1 = fmaxf(best1, __shfl_xor_sync(0xFFFFFFFFu, best1, o));
            }
            const uint32_t ok = __ballot_sync(0xFFFFFFFFu, valid);               // page p0 + n: lanes 4 n .. 4 n + 3
            if (lane < 8) {
                const float mine = __shfl_sync(0xFFu, best0, lane >> 1), other = __shfl_sync(0xFFu, best1, lane >> 1);
                const int at = p0 + lane;
                float u = (lane & 1 ? other : mine) * a.scale;
                if (!(ok >> (4 * lane) & 1)) u = -kForced;
                if (at < a.keep_first || at >= pages - a.keep_last) u = kForced;
                if (at < pages) {
                    float* to = a.scores + out_row * a.ld + at;
                    *to = r0 > 0 ? fmaxf(*to, u) : u;
                }
            }
        }
    }
}

}  // namespace

cudaError_t launch_page_scores(const void* bounds, int64_t n_pages, int P, int H_kv, int d, const void* q, int64_t q_stride, int n_step, int group,
                               const int32_t* table, int64_t ld_table, const int32_t* lens, int B, int keep_first, int keep_last, float scale,
                               float* scores, int64_t ld, int32_t* n_out, int sm_count, cudaStream_t stream) {
    ScoreArgsP a{static_cast<const __nv_bfloat16*>(bounds), n_pages, P, H_kv, static_cast<const __nv_bfloat16*>(q), q_stride, n_step, group, table, ld_table,
                 lens, keep_first, keep_last, scale, scores, ld, n_out, 1, 1};
    const bool few = n_step * group <= 16;
    while (few && a.heads < 8 && H_kv % (2 * a.heads) == 0) a.heads *= 2;      // (more rows: q of one head in shared memory)
    // As many groups of eight pages a warp as leave two CTAs for every SM a few times over: requests end anywhere in front of ld_table.
    const int64_t most = ld_table < (1 << 27) ? ld_table : 1 << 27;                  // pages of 2^31 positions
    const int64_t groups = (most + 7) / 8, slices = kWarps / a.heads;
    const int64_t all = (groups + slices - 1) / slices * B * (H_kv / a.heads);      // CTAs with one group a warp
    while (a.groups_per_warp < 8 && all / (a.groups_per_warp + 1) >= 2 * sm_count) ++a.groups_per_warp;
    const int64_t per_cta = slices * a.groups_per_warp;
    const dim3 grid(static_cast<unsigned>((groups + per_cta - 1) / per_cta), static_cast<unsigned>(H_kv / a.heads), static_cast<unsigned>(B));
    if (d == 128)
        return few ? launch_behind(page_scores_kernel<128, true>, grid, kWarps * 32, 0, stream, a)
                   : launch_behind(page_scores_kernel<128, false>, grid, kWarps * 32, 0, stream, a);
    return few ? launch_behind(page_scores_kernel<64, true>, grid, kWarps * 32, 0, stream, a)
               : launch_behind(page_scores_kernel<64, false>, grid, kWarps * 32, 0, stream, a);
}

}  // namespace idxc
