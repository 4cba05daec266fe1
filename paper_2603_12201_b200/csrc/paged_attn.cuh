// What the kernels of attention over a paged cache share: the call's parameters, the cut of its work into runs, and the merge of segments that runs cut.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "kernels.h"
#include "ptx_sm100.cuh"

namespace idxc {
namespace paged {

constexpr int kSegmentTiles = 4;                // what a segment's beginning and end cost, in tiles
constexpr float kF16Head = 64.f;                // probabilities times scale reach 2^8; f16 holds them times 2^6

struct Params {
    PagedAttnArgs a;
    int heads;                   // key heads that as many neighbouring CTAs walk through in step
    int units;                   // of a request for a CTA: key heads / heads
    int row_blocks;              // blocks of query rows of a (request, key head)
    int tile_log2;               // keys of a tile
    int ways;                    // blocks of 128 rows that share a CTA's tiles (paged_attn_rows.cu)
    int join;                    // 0: runs over all units; else a unit is a cluster's of so many CTAs, which join their parts themselves
    int piece_log2;              // keys of a copy: 16, 32 or 64
    float scale_log2;            // scale * log2(e)
    float* part_o;               // [grid][2][MAXR][D]
    float2* part_ml;             // [grid][2][MAXR] (maximum in log2 units, sum)
    int4* owners;                // [grid] the segment that begins in a CTA's run and does not end in it: (request, key head * row_blocks + block of rows,
                                 // pieces); -1: none
    unsigned int* status;
};

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float ld_shared_f32(uint32_t addr) {
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float2 ld_shared_f32x2(uint32_t addr) {
    float2 v;
    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float4 ld_shared_f32x4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void st_shared_f32(uint32_t addr, float x) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(addr), "f"(x) : "memory"); }
__device__ __forceinline__ void st_shared_f32x2(uint32_t addr, float x, float y) {
    asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(addr), "f"(x), "f"(y) : "memory");
}
// log2 of a positive scale, rounded up, as a number between -60 and 100. (A row's largest probability is 2 to minus that, against the reference that it goes into:
// with 100, probabilities down to 2^-26 of it are normal numbers; with -60, sums of 2^30 of them and the reference's lag stay below 2^98.)
__device__ __forceinline__ float log2_above(float scale) {
    return static_cast<float>(min(max(static_cast<int>(__float_as_uint(scale) >> 23 & 255u) - 126, -60), 100));
}
// Keys of request b that the call knows of.
__device__ __forceinline__ int length_of(const PagedAttnArgs& a, int b) { return min(max(a.lens[b], 0), static_cast<int>(a.max_len)); }
// Tiles of one (key head, block of rows) of request b: of its keys, or of the first min(n_sel, pages of the request) entries of its selection.
__device__ __forceinline__ int tiles_of(const Params& p, int b) {
    const int len = length_of(p.a, b), up = (1 << p.tile_log2) - 1;
    if (!p.a.pages) return (len + up) >> p.tile_log2;
    const int pages = (len + p.a.c.page_size - 1) / p.a.c.page_size;
    return static_cast<int>((static_cast<int64_t>(min(p.a.n_sel, pages)) * p.a.c.page_size + up) >> p.tile_log2);
}
// p.heads neighbouring CTAs take the same stretch of keys for as many key heads, so that the rows of one token, which lie side by side in a cache with
// tokens in front of heads, are read at about the same time (128-byte rows of 8 heads: 5.3 TB/s when every head went its own way). The units
// (request, its heads for this CTA, block of rows) lie end to end, each kSegmentTiles and its tiles long, and are cut into runs of equal length: a
// run with many short segments gets fewer tiles. A run that ends among the first kSegmentTiles of a unit has none of its tiles.
struct Run {
    int b, x;             // request, place among all of the request's units
    int n;                // length
    int total;            // of all units
};
__device__ __forceinline__ int length_of_unit(int tiles) { return tiles > 0 ? tiles + kSegmentTiles : 0; }
// Beginning of a CTA's run: total * cta / n, cut among n = min(grid, total) CTAs so that no run in front of another is empty.
__device__ __forceinline__ int run_begin(int total, int cta, int grid) {
    const int n = min(grid, total);
    if (cta >= n) return total;
    const unsigned each = static_cast<unsigned>(total) / n, more = total - each * n;
    return static_cast<int>(each * cta + more * cta / n);
}
// length(b): of all of request b's units. (At most 16 warps.)
template <class F>
__device__ __forceinline__ Run find_run(const Params& p, int* scratch /* shared, 18 words */, const F& length) {
    const int cta = blockIdx.x / p.heads, ctas = gridDim.x / p.heads;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_thr = blockDim.x, n_warps = n_thr >> 5;
    int sum = 0, mine = 0;
    for (int b = threadIdx.x; b < p.a.B; b += n_thr) {
        const int n = length(b);
        if (b < n_thr) mine = n;
        sum += n;
    }
    sum = __reduce_add_sync(0xFFFFFFFFu, sum);
    if (lane == 0) scratch[warp] = sum;
    __syncthreads();
    Run r{0, 0, 0, 0};
    for (int w = 0; w < n_warps; ++w) r.total += scratch[w];
    const int first = run_begin(r.total, cta, ctas);
    r.n = run_begin(r.total, cta + 1, ctas) - first;
    if (r.n > 0) {                               // (uniform over the CTA)
        int before_block = 0;
        for (int b0 = 0; b0 < p.a.B; b0 += n_thr) {
            const int b = b0 + threadIdx.x;
            const int n = b0 == 0 ? mine : (b < p.a.B ? length(b) : 0);
            int incl = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xFFFFFFFFu, incl, o);
                if (lane >= o) incl += y;
            }
            __syncthreads();
            if (lane == 31) scratch[warp] = incl;
            __syncthreads();
            int before = before_block + incl - n, all = 0;
            for (int w = 0; w < n_warps; ++w) {
                if (w < warp) before += scratch[w];
                all += scratch[w];
            }
            if (first >= before && first < before + n) {
                scratch[16] = b;
                scratch[17] = first - before;
            }
            before_block += all;
            if (first < before_block) break;
        }
        __syncthreads();
        r.b = scratch[16];
        r.x = scratch[17];
    }
    return r;
}
struct Segment {
    int b, head;          // request, key head
    int rows;             // block of query rows
    int t0, n, nt;        // first tile, tiles here, tiles of the unit
};
// Runs over which a segment goes that begins in this CTA's and does not end in it: the tiles that are left lie in the runs that follow.
__device__ __forceinline__ int pieces_of(const Run& run, const Segment& s, int heads) {
    const int cta = blockIdx.x / heads, ctas = min(static_cast<int>(gridDim.x) / heads, run.total);
    const int last_tile = run_begin(run.total, cta + 1, ctas) + (s.nt - s.n) - 1;                              // its place; it is in the run of the
    const int last = static_cast<int>(((static_cast<int64_t>(last_tile) + 1) * ctas + run.total - 1) / run.total) - 1;      // last c with total * c / ctas <= last_tile
    return last - cta + 1;
}

// Joins the pieces of a segment that runs cut. blockIdx.x: the CTA in whose run the segment begins; kMergeWarps warps a row, which take its pieces in turn. Two
// round trips to memory: the owner's word, then maxima, sums and the first pieces together. Units of many pieces get four warps a row (a request of 36392
// keys and one key head has 296: 37 us in all with one warp, 18 with four), others one (96 requests of 2000 positions, 36 us in all, and 47 with four).
template <int D, int ROWS, int kMergeWarps, int kMergeRows>
__global__ void __launch_bounds__(32 * kMergeWarps * kMergeRows)
paged_merge_kernel(const __grid_constant__ Params p, float out_scale) {
    __shared__ float acc_s[kMergeRows][kMergeWarps][D], sum_s[kMergeRows][kMergeWarps];
    let_next_start();
    wait_for_previous();
    const int4 own = p.owners[blockIdx.x];
    if (own.x < 0) return;
    const int lane = threadIdx.x & 31, sub = (threadIdx.x >> 5) % kMergeWarps, in = (threadIdx.x >> 5) / kMergeWarps, r = blockIdx.y * kMergeRows + in;
    const int head = own.y / p.row_blocks, row0 = (own.y - head * p.row_blocks) * ROWS, pieces = own.z;
    const int n_rows = min(p.a.n_step * p.a.group - row0, ROWS);
    const bool works = r < n_rows;
    constexpr int V = D / 32, AHEAD = 4;         // columns of a lane; pieces on their way at a time
    auto row_of = [&](int i) -> int64_t { return (static_cast<int64_t>(blockIdx.x + i * p.heads) * 2 + (i == 0 ? 1 : 0)) * ROWS + r; };
    auto load = [&](int i, float(&y)[V]) {
        const float* from = p.part_o + row_of(i) * D + lane * V;
        if (V == 4) {
            const float4 z = *reinterpret_cast<const float4*>(from);
            y[0] = z.x;
            y[1] = z.y;
            y[2 % V] = z.z;
            y[3 % V] = z.w;
        } else {
            const float2 z = *reinterpret_cast<const float2*>(from);
            y[0] = z.x;
            y[1] = z.y;
        }
    };
    const int mine = works && sub < pieces ? (pieces - sub + kMergeWarps - 1) / kMergeWarps : 0;      // this warp's: sub, sub + kMergeWarps, ...
    float y[AHEAD][V];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
        if (u < mine) load(sub + u * kMergeWarps, y[u]);
    float top = -INFINITY;
    if (works)
        for (int i = lane; i < pieces; i += 32) top = fmaxf(top, p.part_ml[row_of(i)].x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    const float use = top == -INFINITY ? 0.f : top;
    float acc[V] = {}, sum = 0.f;
    for (int i0 = 0; i0 < mine; i0 += 32) {
        float w = 0.f, lw = 0.f;
        if (i0 + lane < mine) {
            const float2 ml = p.part_ml[row_of(sub + (i0 + lane) * kMergeWarps)];
            w = exp2_fast(ml.x - use);
            lw = w * ml.y;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) lw += __shfl_xor_sync(0xFFFFFFFFu, lw, o);
        sum += lw;
        const int n = min(32, mine - i0);
        for (int i = 0; i < n; i += AHEAD) {
            float z[AHEAD][V];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
#pragma unroll
                for (int v = 0; v < V; ++v) z[u][v] = y[u][v];
                if (i0 + i + AHEAD + u < mine) load(sub + (i0 + i + AHEAD + u) * kMergeWarps, y[u]);
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const float wi = __shfl_sync(0xFFFFFFFFu, w, i + u);
                if (i + u < n) {
#pragma unroll
                    for (int v = 0; v < V; ++v) acc[v] += wi * z[u][v];
                }
            }
        }
    }
    if (kMergeWarps > 1) {
#pragma unroll
        for (int v = 0; v < V; ++v) acc_s[in][sub][lane * V + v] = acc[v];
        if (lane == 0) sum_s[in][sub] = sum;
        __syncthreads();
    }
    if (sub != 0 || !works) return;
    for (int w = 1; w < kMergeWarps; ++w) {
        sum += sum_s[in][w];
#pragma unroll
        for (int v = 0; v < V; ++v) acc[v] += acc_s[in][w][lane * V + v];
    }
    const float over = sum == 0.f ? 0.f : out_scale / sum;
    const int step = (row0 + r) / p.a.group, h = row0 + r - step * p.a.group;
    const int64_t row = (static_cast<int64_t>(own.x) * p.a.n_step + step) * p.a.H + head * p.a.group + h;
    __nv_bfloat16* to = p.a.out + row * D + lane * V;
    if (V == 4) *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16(acc[0] * over, acc[1] * over), pack_bf16(acc[2 % V] * over, acc[3 % V] * over));
    else *reinterpret_cast<uint32_t*>(to) = pack_bf16(acc[0] * over, acc[1] * over);
    if (p.a.lse && lane == 0) p.a.lse[row] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
}

}  // namespace paged
}  // namespace idxc
