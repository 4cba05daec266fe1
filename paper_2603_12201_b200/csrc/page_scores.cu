// The largest score that any key of a page could reach, from the page's bounds lo_d <= k_d <= hi_d:
//     u[b, g, p] = scale * max over the new tokens and heads of key head g of  sum_d max(q_d lo_d, q_d hi_d)
// With q = q+ + q- (its positive and its negative part) the sum is <q+, hi> + <q-, lo>: a matrix product over 2 d columns, q's rows against the
// pages' bounds as they lie in memory, in bf16 with fp32 accumulation (the parts of q are exact). Each bound is read once, 4 d bytes a page and
// head, for 4 d flops a query row: HBM-bound for the 1 to 64 rows of a decode step. A page's bounds lie side by side over the heads: a bulk copy brings
// those of up to eight heads of a page (4 KB) into a ring in shared memory, 64 (page, head) pairs a stage; eight warps take eight pages of a head each
// with warp-level MMAs (rows as M, pages as N). The columns are permuted alike in both operands, so that a lane's share of four fragments is 16
// contiguous bytes, and slots lie 64 bytes farther apart than they are long, so that the reads meet no bank twice. 32 requests of 8K to 64K positions
// (73702 pages of 8 heads, d = 128): 54 us, 5.6 TB/s; with fragments straight from global memory, 64 bytes of eight pages an instruction, 58 where this took 53.
//
// A key of -inf in a column where q is positive must not hide its page: the products with the part of q that is 0 are 0 * -inf then, and the sum is no
// number. So are sums with a q that holds none. Such sums are carried through every maximum, and those pages (none, as a rule) are scored again column by column.
#include <cuda_bf16.h>

#include "kernels.h"
#include "ptx_sm100.cuh"

namespace idxc {
namespace {

constexpr int kWarps = 8;                        // a ninth is the producer
constexpr int kMaxRows = 64;                     // query rows of a launch (more: 8 x 32768 positions 54 us a launch, 2048 rows 1.7 ms)
constexpr int kStages = 3;
constexpr float kForced = 3.0e38f;

struct ScoreArgsP {
    const __nv_bfloat16* bounds;
    int64_t n_pages;
    int P, H_kv;
    const __nv_bfloat16* q;
    int64_t q_stride;            // elements between the tokens of q
    int n_step, group;
    int row0, rows;              // query rows of this launch; with row0 > 0 the scores are raised, not set
    const int32_t* table;
    int64_t ld_table;
    const int32_t* lens;
    int keep_first, keep_last;
    float scale;
    float* scores;
    int64_t ld;
    int32_t* n_out;
    int steps;                   // stages' worth of pages a CTA takes: at most 8
    int heads;                   // key heads of a CTA: 1, 2, 4 or 8
    unsigned int* status;
};

template <bool POSITIVE>
__device__ __forceinline__ uint32_t part_of(uint32_t x) {
    uint32_t r;
    if (POSITIVE) asm volatile("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(0u));
    else asm volatile("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(0u));
    return r;
}
// The larger one; none if either is none.
__device__ __forceinline__ float max_or_none(float x, float y) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
    return r;
}
// One page's score by its definition, for a warp: `edge` the bounds of a page and head, `first` the token of the launch's first query row, `h` that row's place among
// the key head's, whose first head q points to. A product of 0 and an infinity is 0; a row whose sum is no number scores kForced.
template <int D>
__device__ __noinline__ float score_by_columns(const __nv_bfloat16* edge, const __nv_bfloat16* q, int64_t q_stride, int group, int first, int h, int rows,
                                               float scale) {
    constexpr int V = D / 32;
    const int at = (threadIdx.x & 31) * V;
    auto product = [](float x, float y) { return (x == 0.f && fabsf(y) == INFINITY) || (y == 0.f && fabsf(x) == INFINITY) ? 0.f : x * y; };
    float best = -INFINITY;
    for (int r = 0; r < rows; ++r) {
        float sum = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float x = __bfloat162float(q[first * q_stride + h * D + at + v]);
            sum += max_or_none(product(x, __bfloat162float(edge[at + v])), product(x, __bfloat162float(edge[D + at + v])));
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        best = fmaxf(best, sum == sum ? sum * scale : kForced);
        if (++h == group) {
            h = 0;
            ++first;
        }
    }
    return best;
}

template <int D>
constexpr int kStageBytes = 64 * 4 * D + 64 * 64;            // 64 (page, head) pairs; at most 64 slots, each 64 bytes longer than its pairs
template <int D>
constexpr int kScoreSmem = kStages * kStageBytes<D>;

// FEW: at most 16 query rows; their fragments stay in registers.
template <int D, bool FEW>
__global__ void __launch_bounds__((kWarps + 1) * 32, 2)
page_scores_kernel(const ScoreArgsP a) {
    constexpr int KC = D / 32;                   // 64-byte pieces of a row of d columns
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ uint4 q_smem[FEW ? 1 : kMaxRows * D / 8];
    __shared__ uint64_t bars[2 * kStages];
    __shared__ uint32_t valid_s[kStages][2];     // which of a stage's pages are the cache's
    __shared__ uint32_t abort_word;
    volatile uint32_t* abort_flag = &abort_word;
    const uint32_t ring_s = smem_u32(ring), full = smem_u32(bars), empty = full + 8 * kStages;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, j = lane & 3;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, kWarps);
        }
        abort_word = 0;
        fence_mbar_init();
    }
    let_next_start();
    wait_for_previous();
    const int b = blockIdx.z, slices = kWarps / a.heads, per_step = 8 * slices;
    const int64_t len = max(a.lens[b], 0);
    const int pages = static_cast<int>(min((len + a.P - 1) / a.P, a.ld_table));
    if (blockIdx.x == 0 && threadIdx.x < a.heads) a.n_out[static_cast<int64_t>(b) * a.H_kv + blockIdx.y * a.heads + threadIdx.x] = pages;
    const int64_t from = static_cast<int64_t>(blockIdx.x) * a.steps * per_step;
    if (from >= pages) return;
    const int first = static_cast<int>(from), n = min(a.steps, (pages - first + per_step - 1) / per_step);
    const uint32_t slot_bytes = a.heads * 4 * D + 64;
    __syncthreads();                             // (the barriers)

    if (warp == kWarps) {
        // ------------------------------------------------------------ producer: a page's bounds of the CTA's heads a copy
        const int32_t* table = a.table + b * a.ld_table;
        auto page_of = [&](int i, int h) -> int {                 // of slot 32 h + lane of step i; -1: none
            const int slot = 32 * h + lane, p = first + i * per_step + slot;
            return i < n && slot < per_step && p < pages ? table[p] : -1;
        };
        int next[2] = {page_of(0, 0), page_of(0, 1)};
        for (int i = 0; i < n; ++i) {
            const int now[2] = {next[0], next[1]};
            next[0] = page_of(i + 1, 0);
            next[1] = page_of(i + 1, 1);
            const int st = i % kStages;
            if (i >= kStages && !mbar_wait(empty + 8 * st, ((i / kStages) & 1) ^ 1, abort_flag)) {
                if (lane == 0) {
                    *abort_flag = 1;
                    atomicCAS(a.status, DEV_OK, DEV_TIMEOUT_PRODUCER);
                }
                for (int k = i - kStages; k < i; ++k) {           // its own copies land before it leaves
                    const long long t0 = clock64();
                    while (!mbar_try_wait(full + 8 * (k % kStages), (k / kStages) & 1) && clock64() - t0 < kWaitCycleBudget) {}
                }
                return;
            }
            bool ok[2];
            uint32_t who[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                ok[h] = now[h] >= 0 && now[h] < a.n_pages;
                who[h] = __ballot_sync(0xFFFFFFFFu, ok[h]);
            }
            if (lane == 0) {
                valid_s[st][0] = who[0];
                valid_s[st][1] = who[1];
                mbar_arrive_expect_tx(full + 8 * st, (__popc(who[0]) + __popc(who[1])) * (slot_bytes - 64));
            }
            __syncwarp();
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (ok[h])
                    bulk_load_1d(ring_s + st * kStageBytes<D> + (32 * h + lane) * slot_bytes,
                                 a.bounds + (static_cast<int64_t>(now[h]) * a.H_kv + blockIdx.y * a.heads) * 2 * D, slot_bytes - 64, full + 8 * st);
        }
        return;
    }

    // ---------------------------------------------------------------- consumers
    const int head = blockIdx.y * a.heads + warp % a.heads, slice = warp / a.heads;
    float* out = a.scores + (static_cast<int64_t>(b) * a.H_kv + head) * a.ld;
    auto q_row = [&](int r) -> const uint4* {    // query row row0 + r: its token, and its head among the key head's
        const int i = (a.row0 + r) / a.group, h = a.row0 + r - i * a.group;
        return reinterpret_cast<const uint4*>(a.q + (static_cast<int64_t>(b) * a.n_step + i) * a.q_stride + static_cast<int64_t>(head * a.group + h) * D);
    };
    const uint4 none = make_uint4(0u, 0u, 0u, 0u);
    const int tiles = FEW ? 1 : (a.rows + 15) / 16;
    uint4 qa[FEW ? KC : 1], qb[FEW ? KC : 1];    // rows g and g + 8
    if (FEW) {
#pragma unroll
        for (int c = 0; c < KC; ++c) {
            qa[FEW ? c : 0] = g < a.rows ? q_row(g)[4 * c + j] : none;
            qb[FEW ? c : 0] = g + 8 < a.rows ? q_row(g + 8)[4 * c + j] : none;
        }
    } else {                                     // (one head a CTA)
        for (int i = threadIdx.x; i < tiles * 16 * (D / 8); i += kWarps * 32) {
            const int r = i / (D / 8), c = i - r * (D / 8);
            q_smem[FEW ? 0 : r * (D / 8) + (c ^ (r & 7))] = r < a.rows ? q_row(r)[c] : none;
        }
        asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");
    }
    uint32_t again = 0;                          // steps whose page of this lane has to be scored column by column
    for (int i = 0; i < n; ++i) {
        const int st = i % kStages, p0 = first + i * per_step + slice * 8;
        if (!mbar_wait(full + 8 * st, (i / kStages) & 1, abort_flag)) {
            if (lane == 0) {
                *abort_flag = 1;
                atomicCAS(a.status, DEV_OK, DEV_TIMEOUT_EPILOGUE);
            }
            return;
        }
        const uint32_t ok = valid_s[st][slice >> 2] >> (8 * (slice & 3));      // pages p0 + 0 .. 7
        const uint32_t at = ring_s + st * kStageBytes<D> + (slice * 8 + g) * slot_bytes + (warp % a.heads) * 4 * D + j * 16;
        uint4 lo[KC], hi[KC];
#pragma unroll
        for (int c = 0; c < KC; ++c) {
            lo[c] = ld_shared_v4(at + c * 64);
            hi[c] = ld_shared_v4(at + 2 * D + c * 64);
        }
        fence_proxy_async_smem();                // (the loads may still be under way, and the next copy is the asynchronous proxy's)
        __syncwarp();
        if (lane == 0) mbar_arrive(empty + 8 * st);
        float best0 = -INFINITY, best1 = -INFINITY;                // pages p0 + 2 j, + 1
        for (int t = 0; t < tiles; ++t) {
            float acc[4] = {0.f, 0.f, 0.f, 0.f}, more[4] = {0.f, 0.f, 0.f, 0.f};
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
                mma_16816<false>(more, h0, hi[c].x, hi[c].y);
                mma_16816<false>(acc, l1, lo[c].z, lo[c].w);
                mma_16816<false>(more, h1, hi[c].z, hi[c].w);
            }
            const int r = t * 16 + g;
            if (r < a.rows) {
                best0 = max_or_none(best0, acc[0] + more[0]);
                best1 = max_or_none(best1, acc[1] + more[1]);
            }
            if (r + 8 < a.rows) {
                best0 = max_or_none(best0, acc[2] + more[2]);
                best1 = max_or_none(best1, acc[3] + more[3]);
            }
        }
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
            best0 = max_or_none(best0, __shfl_xor_sync(0xFFFFFFFFu, best0, o));
            best1 = max_or_none(best1, __shfl_xor_sync(0xFFFFFFFFu, best1, o));
        }
        const float mine = __shfl_sync(0xFFFFFFFFu, best0, (lane >> 1) & 3), other = __shfl_sync(0xFFFFFFFFu, best1, (lane >> 1) & 3);
        const int p = p0 + lane;
        if (lane < 8 && p < pages) {
            float u = (lane & 1 ? other : mine) * a.scale;
            if (!(ok >> lane & 1)) u = -kForced;
            if (p < a.keep_first || p >= pages - a.keep_last) u = kForced;
            if (u != u) again |= 1u << i;
            else out[p] = a.row0 > 0 ? fmaxf(out[p], u) : u;
        }
    }
    if (!__any_sync(0xFFFFFFFFu, again != 0u)) return;
    for (int i = 0; i < n; ++i)
        for (uint32_t none = __ballot_sync(0xFFFFFFFFu, again >> i & 1u); none; none &= none - 1) {
            const int p = first + i * per_step + slice * 8 + __ffs(none) - 1, token = a.row0 / a.group;
            const int64_t page = a.table[b * a.ld_table + p];
            const float u = score_by_columns<D>(a.bounds + (page * a.H_kv + head) * 2 * D,
                                                a.q + static_cast<int64_t>(b) * a.n_step * a.q_stride + static_cast<int64_t>(head) * a.group * D, a.q_stride, a.group, token,
                                                a.row0 - token * a.group, a.rows, a.scale);
            if (lane == 0) out[p] = a.row0 > 0 ? fmaxf(out[p], u) : u;
        }
}

template <int D, bool FEW>
cudaError_t run(const ScoreArgsP& a, dim3 grid, cudaStream_t stream) {
    const cudaError_t e = ensure_max_dynamic_smem(reinterpret_cast<const void*>(page_scores_kernel<D, FEW>), kScoreSmem<D>);
    return e != cudaSuccess ? e : launch_behind(page_scores_kernel<D, FEW>, grid, (kWarps + 1) * 32, kScoreSmem<D>, stream, a);
}

}  // namespace

cudaError_t launch_page_scores(const void* bounds, int64_t n_pages, int P, int H_kv, int d, const void* q, int64_t q_stride, int n_step, int group,
                               const int32_t* table, int64_t ld_table, const int32_t* lens, int B, int keep_first, int keep_last, float scale,
                               float* scores, int64_t ld, int32_t* n_out, unsigned int* status, int sm_count, cudaStream_t stream, int* launches) {
    ScoreArgsP a{static_cast<const __nv_bfloat16*>(bounds), n_pages, P, H_kv, static_cast<const __nv_bfloat16*>(q), q_stride, n_step, group, 0, 0, table,
                 ld_table, lens, keep_first, keep_last, scale, scores, ld, n_out, 1, 1, status};
    const int rows = n_step * group;
    const bool few = rows <= 16;
    while (few && a.heads < 8 && H_kv % (2 * a.heads) == 0) a.heads *= 2;      // (more rows: q of one head in shared memory)
    // Steps of a CTA: as many as leave two CTAs for every SM, up to 8. (The same 32 requests, which end anywhere in front of ld_table: 75, 58, 53, 57 and
    // 63 us with at most 2, 4, 8, 16 and 32.)
    const int64_t most = ld_table < (1 << 27) ? ld_table : 1 << 27;            // pages of 2^31 positions
    const int per_step = 8 * (kWarps / a.heads);
    const int64_t steps = (most + per_step - 1) / per_step;
    while (a.steps < 8 && steps * B * (H_kv / a.heads) / (a.steps + 1) >= 2 * sm_count) ++a.steps;
    const dim3 grid(static_cast<unsigned>(steps > 0 ? (steps + a.steps - 1) / a.steps : 1), static_cast<unsigned>(H_kv / a.heads), static_cast<unsigned>(B));
    for (a.row0 = 0; a.row0 < rows; a.row0 += kMaxRows) {
        a.rows = rows - a.row0 < kMaxRows ? rows - a.row0 : kMaxRows;
        *launches += 1;
        const cudaError_t e = d == 128 ? (few ? run<128, true>(a, grid, stream) : run<128, false>(a, grid, stream))
                                       : (few ? run<64, true>(a, grid, stream) : run<64, false>(a, grid, stream));
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace idxc
