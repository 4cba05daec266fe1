// Head-summed attention weights over latent cache rows: for every cached position s of a sequence
//     acc[b, s] = beta acc[b, s] + sum_r exp(scale <q_r, row_s> - lse_r)        r = (new token, head)
// A score product with an exponential and a row sum behind it, no second product. The cache rows are the M of the MMAs (128 a tile), the
// query rows the N, so a thread of the epilogue owns one position and sums over its accumulator row: no exchange between
// threads, one writer per entry (of a selection's entries that name a position again each adds the same number: same row, same order of
// every sum). Q stays in shared memory; the row blocks [128 rows x 128 B] stream through a ring of four, so
// a tile's scores start with its first 64 columns. HBM-bound with bf16 rows: 64 KB of the ring in flight per SM; the MMAs of a tile take
// 2300 clocks at 128 query rows (64 each), the bytes of a tile 6400 at the copy rate.
// bf16 rows of a sequence come by TMA, selected bf16 rows by 16-byte asynchronous copies, 4-bit rows through the registers of eight warps.
// More than 128 query rows a sequence: one launch per 128, each of which reads the rows and the sums again (8 x 40K bf16 rows, 128 heads: 75 us
// for one new token, 297 us for four, 2.4 ms for 32; read once, the bytes and products of four would take 123 us).
// Selected bf16 rows: the four warps of a set wait for a block's copies before they ask for their next one, so a set has one block on its way (32
// selections of 2048 rows, 128 heads: 28 us, 24 us over 4-bit rows; their bytes alone 12 and 6 us).
#include "latent_attn.cuh"

namespace idxc {
using namespace latent;
namespace {

constexpr int kWTile = 128;                          // cache rows of a tile (2^7)
constexpr int kWRows = 128;                          // query rows of a launch at most
constexpr int kRing = 4;
constexpr uint32_t kRingBytes = kWTile * 128;
constexpr uint32_t kQMax = kBlocks * kWRows * 128;
constexpr uint32_t kTabBytes = 4 * kWRows * 8;       // per epilogue warp: lse in log2 units, and the keys that each query row sees
constexpr uint32_t kWBarBytes = 256;
constexpr uint32_t kWSmemBytes = kQMax + kRing * kRingBytes + kTabBytes + kWBarBytes + 1024;
static_assert(kWSmemBytes <= 232448, "shared memory of a CTA");
enum Source { kTma, kCopy, kCodes };                 // bf16 rows in order, selected bf16 rows, 4-bit rows

struct WParams {
    LatentArgs a;
    UnitTiles tiles;
    uint32_t units;              // sequences
    int groups;
    int row0, rows;              // query rows row0 .. row0 + rows - 1 of every sequence
    uint32_t n;                  // rows rounded up to 16: the N of the MMAs
    float scale_log2;
    const float* lse;
    float beta;
    float* acc;
    int64_t ld;
    unsigned int* status;
};

// cache row of entry j of sequence b, -1: none
__device__ __forceinline__ int entry_row(const LatentArgs& a, int64_t b, int64_t base, int j, int len) {
    if (j >= len) return -1;
    int64_t r = j;
    if (a.topk) {
        r = __ldg(a.topk + b * a.k_top + j);
        if (r < 0) return -1;
    }
    r += base;
    return r >= 0 && r < a.n_kv ? static_cast<int>(r) : -1;
}

template <Source SRC>
__global__ void __launch_bounds__(SRC == kTma ? 256 : 512, 1)
attn_weights_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap kv_map, const WParams p) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint8_t* q_smem = smem;
    uint8_t* ring = smem + kQMax;
    float* tab = reinterpret_cast<float*>(ring + kRing * kRingBytes);
    uint64_t* bars = reinterpret_cast<uint64_t*>(ring + kRing * kRingBytes + kTabBytes);
    const uint32_t bar_q_full = smem_u32(bars + 0);
    const uint32_t bar_q_empty = smem_u32(bars + 1);
    const uint32_t bar_full = smem_u32(bars + 2);            // [4]
    const uint32_t bar_empty = smem_u32(bars + 6);           // [4]
    const uint32_t bar_s_full = smem_u32(bars + 10);         // [2]
    const uint32_t bar_s_free = smem_u32(bars + 12);         // [2]
    uint32_t* tmem_base_slot = reinterpret_cast<uint32_t*>(bars + 14);
    volatile uint32_t* abort_flag = tmem_base_slot + 1;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int seq_rows = p.a.n_step * p.a.H;
    auto seq_len = [&](uint32_t b) -> int {
        return p.a.topk ? p.a.k_top : static_cast<int>(min(max(static_cast<int64_t>(__ldg(p.a.lens + b)), int64_t(0)), p.a.max_len));
    };
    auto seq_base = [&](uint32_t b) -> int64_t { return first_row(p.a, b); };

    const EarlyTiles early = early_tiles(p.units, p.tiles);
    early_bases(p.a.kv_base, p.a.B);
    if (threadIdx.x == 0) {
        mbar_init(bar_q_full, 1);
        mbar_init(bar_q_empty, 1);
        for (int i = 0; i < kRing; ++i) {
            mbar_init(bar_full + 8 * i, SRC == kTma ? 1 : 4);
            mbar_init(bar_empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar_s_full + 8 * i, 1);
            mbar_init(bar_s_free + 8 * i, 4);
        }
        *abort_flag = 0u;
        fence_mbar_init();
    }
    if (warp == 0) {
        tmem_alloc(smem_u32(tmem_base_slot), 256);
        tmem_relinquish_alloc_permit();
    }
    tcgen05_fence_before_sync();
    const Run run = find_run(p.units, p.tiles, early, blockIdx.x, p.groups, 0, reinterpret_cast<int*>(tab));
    __syncthreads();
    tcgen05_fence_after_sync();
    const uint32_t tmem_base = *tmem_base_slot;

    Walk walk(p.tiles, run);
    Piece pc{};
    bool ok = true;
    uint32_t tile = 0, item = 0, blk = 0;      // counted over the whole kernel; blk: column blocks (ring slot blk % 4)
    auto give_up = [&](unsigned int code) {
        *abort_flag = 1u;
        atomicCAS(p.status, 0u, code);
    };
    auto wait_warp = [&](uint32_t bar, uint32_t parity) -> bool { return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, abort_flag)); };

    if (warp == 0) {
        // ------------------------------------------------------------ scores
        const uint32_t idesc = umma_idesc(1, 1, kWTile, p.n);
        const uint64_t q_desc = umma_smem_desc_sw128(smem_u32(q_smem)), r_desc = umma_smem_desc_sw128(smem_u32(ring));
        const uint32_t q_block = p.n * 128 / 16;
        while (ok && walk.next(pc)) {
            ok = wait_warp(bar_q_full, item & 1u);
            for (int i = 0; __all_sync(0xFFFFFFFFu, ok && i < pc.n); ++i, ++tile) {
                const uint32_t st = tile & 1u;
                ok = wait_warp(bar_s_free + 8 * st, ((tile >> 1) & 1u) ^ 1u);
                if (!ok) break;
                tcgen05_fence_after_sync();
                uint64_t b_desc = q_desc;
#pragma unroll 1
                for (int b = 0; b < kBlocks; ++b, ++blk) {
                    const uint32_t slot = blk & 3u;
                    ok = wait_warp(bar_full + 8 * slot, (blk >> 2) & 1u);
                    if (!ok) break;
                    umma_f16_x4<2, 2>(tmem_base + st * 128, r_desc + slot * (kRingBytes / 16), b_desc, idesc, b != 0 ? 1u : 0u);
                    umma_commit_elect(bar_empty + 8 * slot);
                    b_desc += q_block;
                }
                if (!ok) break;
                umma_commit_elect(bar_s_full + 8 * st);
            }
            if (ok) umma_commit_elect(bar_q_empty);
            ++item;
        }
        if (!ok && lane == 0) give_up(DEV_TIMEOUT_MMA);
    } else if (warp == 2) {
        // ------------------------------------------------------------ Q
        if (lane == 0) {
            tma_prefetch_desc(&q_map);
            int before = 0;                                  // tiles of the piece before
            while (ok && walk.next(pc)) {
                ok = mbar_wait(bar_q_empty, (item & 1u) ^ 1u, abort_flag, piece_budget(before), 200);
                before = pc.n;
                if (!ok) break;
                mbar_arrive_expect_tx(bar_q_full, kBlocks * p.n * 128);
                for (int b = 0; b < kBlocks; ++b)
                    tma_load_2d(smem_u32(q_smem + b * p.n * 128), &q_map, bar_q_full, b * 64, static_cast<int>(static_cast<int64_t>(pc.unit) * seq_rows + p.row0));
                ++item;
            }
            if (!ok) give_up(DEV_TIMEOUT_PRODUCER);
        }
    } else if (SRC == kTma && warp == 1) {
        // ------------------------------------------------------------ bf16 rows in order. Rows behind the sequence's end only reach sums that nobody writes.
        if (lane == 0) {
            tma_prefetch_desc(&kv_map);
            while (ok && walk.next(pc)) {
                const int64_t base = seq_base(pc.unit);
                for (int i = 0; i < pc.n && ok; ++i) {
                    const int first = static_cast<int>(min(max(base + static_cast<int64_t>(pc.t0 + i) * kWTile, static_cast<int64_t>(-kWTile)), p.a.n_kv));
                    for (int b = 0; b < kBlocks; ++b, ++blk) {
                        const uint32_t slot = blk & 3u;
                        ok = mbar_wait(bar_empty + 8 * slot, ((blk >> 2) & 1u) ^ 1u, abort_flag);
                        if (!ok) break;
                        mbar_arrive_expect_tx(bar_full + 8 * slot, kRingBytes);
                        tma_load_2d(smem_u32(ring + slot * kRingBytes), &kv_map, bar_full + 8 * slot, b * 64, first);
                    }
                }
            }
            if (!ok) give_up(DEV_TIMEOUT_GATHER);
        }
    } else if (SRC != kTma && warp >= 8) {
        // ------------------------------------------------------------ selected or 4-bit rows: two sets of four warps fill the ring's slots in turn
        // (block blk goes to set blk % 2), a warp 32 rows of each.
        const uint32_t set = static_cast<uint32_t>(warp - 8) >> 2;
        const int w = warp & 3;
        const uint8_t* kv = static_cast<const uint8_t*>(p.a.kv);
        const uint32_t ring_addr = smem_u32(ring);
        while (ok && walk.next(pc)) {
            const int64_t base = seq_base(pc.unit);
            const int len = seq_len(pc.unit);
            for (int i = 0; i < pc.n && ok; ++i) {
                const int src = entry_row(p.a, pc.unit, base, (pc.t0 + i) * kWTile + w * 32 + lane, len);
                const uint8_t* row = kv + static_cast<uint64_t>(static_cast<uint32_t>(max(src, 0))) * (SRC == kCodes ? kLatentQ4RowBytes : kLatentBf16RowBytes);
                // 4-bit rows: the lane has its row's codes of two of its set's blocks in registers ahead of the one it stores
                uint32_t c0[8], c1[8], s0 = 0, s1 = 0;
                const int first = static_cast<int>((blk ^ set) & 1u);        // this set's first block of the tile
                if (SRC == kCodes) {
                    load_nc_256(row + first * 32, src >= 0, c0);
                    s0 = load_nc_32(row + kLatentQ4ScaleOff + first * 4, src >= 0);
                    load_nc_256(row + (first + 2) * 32, src >= 0, c1);
                    s1 = load_nc_32(row + kLatentQ4ScaleOff + (first + 2) * 4, src >= 0);
                }
#pragma unroll 1
                for (int b = first; b < kBlocks; b += 2) {
                    const uint32_t at = blk + b, slot = at & 3u, to = ring_addr + slot * kRingBytes;
                    if (SRC == kCopy) {
                        ok = wait_warp(bar_empty + 8 * slot, ((at >> 2) & 1u) ^ 1u);
                        if (!ok) break;
#pragma unroll
                        for (int k = 0; k < 8; ++k) {                        // 4 rows x 128 bytes an instruction
                            const int r = k * 4 + (lane >> 3), ch = lane & 7;
                            const int from = __shfl_sync(0xFFFFFFFFu, src, r);
                            const uint32_t dst = to + (w * 32 + r) * 128 + ((ch ^ (r & 7)) << 4);
                            if (from >= 0) cp_async_16(dst, kv + static_cast<uint64_t>(static_cast<uint32_t>(from)) * kLatentBf16RowBytes + b * 128 + ch * 16);
                            else st_shared_v4(dst, make_uint4(0, 0, 0, 0));
                        }
                        cp_async_wait_all();
                    } else if (b < 8) {
                        uint4 v[8];
                        const Q4Scale lo = q4_scale_of(s0), hi = q4_scale_of(s0 >> 16);
#pragma unroll
                        for (int k = 0; k < 8; ++k) v[k] = dequant8_q4(c0[k], k < 4 ? lo : hi);
#pragma unroll
                        for (int k = 0; k < 8; ++k) c0[k] = c1[k];
                        s0 = s1;
                        if (b + 4 < 8) {
                            load_nc_256(row + (b + 4) * 32, src >= 0, c1);
                            s1 = load_nc_32(row + kLatentQ4ScaleOff + (b + 4) * 4, src >= 0);
                        }
                        ok = wait_warp(bar_empty + 8 * slot, ((at >> 2) & 1u) ^ 1u);
                        if (!ok) break;
                        const uint32_t dst = to + (w * 32 + lane) * 128 + ((lane & 7) << 4);
#pragma unroll
                        for (int k = 0; k < 8; ++k) st_shared_v4(dst ^ (k << 4), v[k]);
                    } else {
                        ok = wait_warp(bar_empty + 8 * slot, ((at >> 2) & 1u) ^ 1u);
                        if (!ok) break;
                        const uint32_t dst = to + (w * 32 + lane) * 128 + ((lane & 7) << 4);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            uint32_t v[8];
                            load_nc_256(row + kLatentQ4RopeOff + k * 32, src >= 0, v);
                            st_shared_v4(dst ^ (2 * k << 4), make_uint4(v[0], v[1], v[2], v[3]));
                            st_shared_v4(dst ^ ((2 * k + 1) << 4), make_uint4(v[4], v[5], v[6], v[7]));
                        }
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar_full + 8 * slot);
                }
                blk += kBlocks;
            }
        }
        if (!ok && lane == 0) give_up(DEV_TIMEOUT_GATHER);
    } else if (warp >= 4 && warp < 8) {
        // ------------------------------------------------------------ exponentials and sums: one cached position a thread
        const int quarter = warp & 3;
        const uint32_t lane_base = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16);
        float* lse2 = tab + quarter * kWRows;                                // this warp's own copies
        int* sees = reinterpret_cast<int*>(tab + 4 * kWRows) + quarter * kWRows;
        while (ok && walk.next(pc)) {
            const int64_t b = pc.unit;
            const int len = seq_len(pc.unit);
            const int64_t base = seq_base(pc.unit);
            __syncwarp();
            int least = len;                                                 // a row without a log-sum-exp counts nowhere, whatever its scores are
            for (int r = lane; r < kWRows; r += 32) {
                const float v = r < p.rows ? __ldg(p.lse + b * seq_rows + p.row0 + r) : 0.f;
                lse2[r] = v * 1.4426950408889634f;
                sees[r] = v == -INFINITY ? 0 : (p.a.topk ? len : len - (p.a.n_step - 1 - (p.row0 + r) / p.a.H));
                if (r < p.rows) least = min(least, sees[r]);
            }
            const int seen_by_all = __reduce_min_sync(0xFFFFFFFFu, least);
            __syncwarp();
            for (int i = 0; i < pc.n && ok; ++i, ++tile) {
                const uint32_t st = tile & 1u;
                const int j = (pc.t0 + i) * kWTile + quarter * 32 + lane;
                const bool use = entry_row(p.a, b, base, j, len) >= 0;
                const bool tail = __any_sync(0xFFFFFFFFu, j >= seen_by_all);       // some row may not count at some position
                float* dst = p.acc + b * p.ld + j;
                float old = 0.f;
                if (!p.a.topk && j < len && p.beta != 0.f) old = p.beta * *dst;
                ok = wait_warp(bar_s_full + 8 * st, (tile >> 1) & 1u);
                if (!ok) break;
                tcgen05_fence_after_sync();
                float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
                for (int c = 0; c < p.rows; c += 32) {
                    uint32_t s[32];
                    tmem_ld_32x32b_x32(lane_base + st * 128 + c, s);
                    tmem_ld_wait(s);
                    if (c + 32 <= p.rows && !tail) {
#pragma unroll
                        for (int k = 0; k < 32; k += 4) {
                            const float4 l = *reinterpret_cast<const float4*>(lse2 + c + k);
                            sum[0] += exp2_fast(__fmaf_rn(__uint_as_float(s[k]), p.scale_log2, -l.x));
                            sum[1] += exp2_fast(__fmaf_rn(__uint_as_float(s[k + 1]), p.scale_log2, -l.y));
                            sum[2] += exp2_fast(__fmaf_rn(__uint_as_float(s[k + 2]), p.scale_log2, -l.z));
                            sum[3] += exp2_fast(__fmaf_rn(__uint_as_float(s[k + 3]), p.scale_log2, -l.w));
                        }
                    } else {
#pragma unroll
                        for (int k = 0; k < 32; ++k) {
                            const float e = exp2_fast(__fmaf_rn(__uint_as_float(s[k]), p.scale_log2, -lse2[c + k]));
                            if (c + k < p.rows && j < sees[c + k]) sum[k & 3] += e;           // (a query row that is not ours may hold anything)
                        }
                    }
                }
                tcgen05_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_s_free + 8 * st);
                const float w = use ? (sum[0] + sum[1]) + (sum[2] + sum[3]) : 0.f;
                if (!p.a.topk) {
                    if (j < len) *dst = old + w;
                } else if (use) {
                    const int s = __ldg(p.a.topk + b * p.a.k_top + j);
                    if (s < p.ld) atomicAdd(p.acc + b * p.ld + s, w);
                }
            }
        }
        if (!ok && lane == 0) give_up(DEV_TIMEOUT_EPILOGUE);
    }

    // ---------------------------------------------------------------- teardown
    __syncwarp();
    if (*abort_flag) {                       // copies may still be in flight: let them land before the CTA's memory goes
        const long long t0 = clock64();
        while (clock64() - t0 < 2000000LL) __nanosleep(1000);
    }
    tcgen05_fence_before_sync();
    __syncthreads();
    if (warp == 0) {
        tcgen05_fence_after_sync();
        tmem_dealloc(tmem_base, 256);
    }
}

}  // namespace

int attn_weights_rows(int n_step, int H, int row0) {
    const int64_t left = static_cast<int64_t>(n_step) * H - row0;
    return static_cast<int>(left < kWRows ? left : kWRows);
}

cudaError_t launch_attn_weights(const LatentArgs& a, int row0, const float* lse, float beta, float* acc, int64_t ld, const CUtensorMap& q_map,
                                const CUtensorMap& kv_map, unsigned int* status, int sm_count, cudaStream_t stream) {
    const int rows = attn_weights_rows(a.n_step, a.H, row0);
    const int64_t tiles = a.B * ((a.max_len + kWTile - 1) / kWTile);
    const int groups = static_cast<int>(tiles < sm_count ? tiles : sm_count);
    const UnitTiles ut{nullptr, a.lens, a.max_len, 1, 7};
    const WParams p{a, ut, static_cast<uint32_t>(a.B), groups, row0, rows, static_cast<uint32_t>((rows + 15) / 16 * 16), a.scale * 1.4426950408889634f,
                    lse, beta, acc, ld, status};
    auto go = [&](auto kernel, int threads) -> cudaError_t {
        if (cudaError_t e = ensure_max_dynamic_smem(reinterpret_cast<const void*>(kernel), kWSmemBytes); e != cudaSuccess) return e;
        kernel<<<groups, threads, kWSmemBytes, stream>>>(q_map, kv_map, p);
        return cudaGetLastError();
    };
    if (a.q4) return go(attn_weights_kernel<kCodes>, 512);
    if (a.topk || a.n_kv == 0) return go(attn_weights_kernel<kCopy>, 512);        // (no rows at all: nothing is copied)
    return go(attn_weights_kernel<kTma>, 256);
}

}  // namespace idxc
