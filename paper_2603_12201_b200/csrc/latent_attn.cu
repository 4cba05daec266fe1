// Attention over latent cache rows, one shared row per token for all heads (keys = its 576 columns, values = its first 512):
// dense over a sequence's rows held in bf16 or 4 bits, and over a selection of 4-bit rows.
//
// One pass over the rows. A CTA holds 64 query rows (heads x new tokens of one sequence): its fp32 output, 64 x 512, is then
// half of tensor memory, so scores, softmax and both halves of the output are done tile by tile with nothing saved or read
// twice. tcgen05.mma with M = 64 puts row r on TMEM lane 32 (r / 16) + r % 16 (+ 16 with a lane offset of 16, measured), so
// the two 256-column halves of O lie on top of each other in 256 columns. M = 64 issues at half the M = 128 rate (N = 64: 32
// clocks, N = 256: 128), 2176 clocks of tensor pipe per 64-row tile, for one query row as for 64. bf16 rows' bytes take 3270 clocks a tile and
// hide them; 4-bit rows' take 1190 and do not: 8 x 131072 4-bit rows take 249 us with 16 heads and 251 with 64 (bytes 67), bf16 rows with 16 heads
// 226 (bytes 184), and 2047 queries over 2048 selected rows 1.05 ms with 16 heads as with 64. More than 64 query rows take a pair of CTAs
// (latent_attn_pair.cu); what surrounds both kernels, the workspace, the count of selected tiles and the merge, is here.
//
// Work: the tiles of all sequences, laid end to end, are cut into equal runs, one per CTA (pair). A run may start and end
// inside a sequence: such a piece leaves a normalised fp32 result and its log-sum-exp in the workspace, and a merge kernel
// weighs the pieces. A run has at most two of them, so the workspace does not grow with the work. Every CTA works out the
// cuts for itself from the lengths on the device.
//
// Shared memory: Q 9 blocks of [64 rows x 128 B] | 2 stages x 9 blocks of [64 cache rows x 128 B] | P [64 x 128 B], all in the
// 128-byte swizzle. A block of cache rows is at once the K-major B operand of Q K^T and the MN-major B operand of P V. A stage
// is five slots with barriers of their own: slots 0..3 = two blocks each (128 value columns, free again when their part of P V is
// done), slot 4 = the positional block (free when its part of the scores is done). P V goes slot by slot, so that a stage is
// being refilled from its front while its back is still multiplied; the scores of the next tile but one start with the
// positional block and follow the refill. (With two slots a stage the refill was waited for: 5250 clocks a tile.)
// TMEM: O [0, 256), both halves | S double-buffered [256, 320), [320, 384).
// Scores and P V are issued by a warp each, so that a tile's softmax runs under the next tile's scores and neither waits for the
// other's operands.
// bf16 rows come by TMA (the tail of a sequence is cleared in shared memory: rows behind it may hold NaN). 4-bit rows are read
// into registers a tile ahead by eight warps and expanded into the stage (exact, see latent_format.cuh).
#include "latent_attn.cuh"

namespace idxc {
using namespace latent;
namespace {

constexpr int kSlots = 5;                           // slots of a stage: blocks 2s, 2s + 1 for s < 4, block 8
constexpr uint32_t kBlockBytes = kTile * 128;
constexpr uint32_t kStageBytes = kBlocks * kBlockBytes;
constexpr uint32_t kQBytes = kBlocks * kRows * 128;
constexpr uint32_t kPBytes = kRows * 128;
constexpr uint32_t kBarBytes = 512;
constexpr uint32_t kSmemBytes = kQBytes + 2 * kStageBytes + kPBytes + kBarBytes + 1024;
static_assert(kSmemBytes <= 232448, "shared memory of a CTA");
constexpr uint32_t kColS = 256;
constexpr int kWarpsBf16 = 8;                       // 0 scores | 1 P V | 2 Q | 3 rows (TMA) | 4..7 softmax
constexpr int kWarpsQ4 = 16;                        // 0 scores | 1 P V | 2 Q | 3 idle | 4..7 softmax | 8..15 rows
constexpr int kCutTiles = 4;                        // (see find_run) 74 queries of 32 selected tiles: 62 us cut even or apart, 100: 84 us and 103
constexpr int kSlotWarps = 4;                       // warps that fill a slot (4-bit rows)

// ---------------------------------------------------------------- plan
// Selected rows: tiles of query t up to its last usable entry.
constexpr int kCountThreads = 256;
__global__ void __launch_bounds__(kCountThreads)
latent_count_kernel(const LatentArgs a, int32_t* __restrict__ tiles) {
    __shared__ int s_last[kCountThreads / 32];
    let_next_start();
    const int64_t t = blockIdx.x;
    const int64_t base = first_row(a, t);
    const int32_t* row = a.topk + t * a.k_top;
    int last = 0;
    for (int j0 = threadIdx.x; j0 < a.k_top; j0 += 8 * kCountThreads) {          // eight loads under way at a time
        int32_t i[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) i[k] = j0 + k * kCountThreads < a.k_top ? __ldg(row + j0 + k * kCountThreads) : -1;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (i[k] >= 0 && base + i[k] >= 0 && base + i[k] < a.n_kv) last = j0 + k * kCountThreads + 1;
    }
    last = __reduce_max_sync(0xFFFFFFFFu, last);
    if ((threadIdx.x & 31) == 0) s_last[threadIdx.x >> 5] = last;
    __syncthreads();
    if (threadIdx.x < 32) {
        last = __reduce_max_sync(0xFFFFFFFFu, threadIdx.x < kCountThreads / 32 ? s_last[threadIdx.x] : 0);
        if (threadIdx.x == 0) tiles[t] = (last + kTile - 1) / kTile;
    }
}

// ---------------------------------------------------------------- main kernel
template <bool Q4>
__global__ void __launch_bounds__((Q4 ? kWarpsQ4 : kWarpsBf16) * 32, 1)
latent_attn_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap rope_map,
                   const __grid_constant__ CUtensorMap v_map, const Params p) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint8_t* q_smem = smem;
    uint8_t* stage_smem = smem + kQBytes;
    uint8_t* p_smem = stage_smem + 2 * kStageBytes;
    uint64_t* bars = reinterpret_cast<uint64_t*>(p_smem + kPBytes);
    const uint32_t bar_q_full = smem_u32(bars + 0);
    const uint32_t bar_q_empty = smem_u32(bars + 1);
    const uint32_t bar_slot_full = smem_u32(bars + 2);       // [2 stages][kSlots]
    const uint32_t bar_slot_empty = smem_u32(bars + 12);
    const uint32_t bar_s_full = smem_u32(bars + 22);         // [2]
    const uint32_t bar_p_ready = smem_u32(bars + 24);
    const uint32_t bar_pv_done = smem_u32(bars + 25);
    const uint32_t bar_o_free = smem_u32(bars + 26);
    const uint32_t bar_tail = smem_u32(bars + 27);
    const uint32_t bar_s_free = smem_u32(bars + 32);         // [2]
    uint32_t* tmem_base_slot = reinterpret_cast<uint32_t*>(bars + 28);
    volatile uint32_t* abort_flag = tmem_base_slot + 1;
    uint8_t* mask_smem = reinterpret_cast<uint8_t*>(bars + 30);    // [2 stages][8]: bit r of a stage's 64: row r of the tile is usable
    static_assert(34 * 8 <= kBarBytes, "barrier area");

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int group = blockIdx.x;
    const int seq_rows = p.a.n_step * p.a.H;
    // query rows of this CTA in a unit: first row within the sequence, and how many
    auto rows_of = [&](uint32_t unit, int64_t& seq, int& r0) -> int {
        const uint32_t s = p.tiles.seq_of(unit);
        seq = s;
        r0 = static_cast<int>(unit - s * p.blocks_per_seq) * kRows;
        return min(kRows, seq_rows - r0);
    };
    auto seq_len = [&](int64_t seq) -> int64_t {
        return p.a.topk ? p.a.k_top : min(max(static_cast<int64_t>(__ldg(p.a.lens + seq)), int64_t(0)), p.a.max_len);
    };

    let_next_start();                                        // the merge
    EarlyTiles early{};
    if (!p.tiles.counted) early = early_tiles(p.units, p.tiles);
    early_bases(p.a.kv_base, p.a.B);
    if (lane == 0 && warp == 2) tma_prefetch_desc(&q_map);
    if (!Q4 && lane == 0 && warp == 3) {
        tma_prefetch_desc(&rope_map);
        tma_prefetch_desc(&v_map);
    }
    if (threadIdx.x == 0) {
        mbar_init(bar_q_full, 1);
        mbar_init(bar_q_empty, 1);
        for (int i = 0; i < 2 * kSlots; ++i) {
            mbar_init(bar_slot_full + 8 * i, Q4 ? kSlotWarps : 1);
            mbar_init(bar_slot_empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar_s_full + 8 * i, 1);
            mbar_init(bar_s_free + 8 * i, 4);
        }
        mbar_init(bar_p_ready, 4);
        mbar_init(bar_pv_done, 1);
        mbar_init(bar_o_free, 4);
        mbar_init(bar_tail, 1);
        *abort_flag = 0u;
        fence_mbar_init();
    }
    if (warp == 0) {
        tmem_alloc(smem_u32(tmem_base_slot), 512);
        tmem_relinquish_alloc_permit();
    }
    tcgen05_fence_before_sync();
    if (p.tiles.counted) {
        wait_for_previous();
        early = early_tiles(p.units, p.tiles);
    }
    const Run run = find_run(p.units, p.tiles, early, group, p.groups, kCutTiles, reinterpret_cast<int*>(q_smem));      // (Q has not been asked for yet)
    if (threadIdx.x == 0) {
        p.starts[group] = make_int2(static_cast<int>(run.unit), run.t);
        p.runs[group] = run.first;
        if (group == p.groups - 1) p.runs[p.groups] = run.total;
    }
    fence_proxy_async_smem();                                // find_run's words before Q's copy over them
    __syncthreads();
    tcgen05_fence_after_sync();
    const uint32_t tmem_base = *tmem_base_slot;

    Walk walk(p.tiles, run);
    Piece pc{};
    int64_t seq;
    int r0;
    bool ok = true;
    uint32_t tile = 0, item = 0;          // counted over the whole kernel: stages, buffers and phases follow from them
    auto give_up = [&](unsigned int code) {
        *abort_flag = 1u;
        atomicCAS(p.status, 0u, code);
    };
    auto wait_warp = [&](uint32_t bar, uint32_t parity, unsigned sleep_ns = 0) -> bool {
        return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, abort_flag, kWaitCycleBudget, sleep_ns));
    };

    if (warp == 0) {
        // ------------------------------------------------------------ scores (warp-uniform, one elected lane issues)
        constexpr uint32_t kIdescS = umma_idesc(1, 1, kRows, kTile);
        const uint64_t q_desc = umma_smem_desc_sw128(smem_u32(q_smem));
        while (ok && walk.next(pc)) {
            rows_of(pc.unit, seq, r0);
            ok = wait_warp(bar_q_full, item & 1u);
            for (int i = 0; __all_sync(0xFFFFFFFFu, ok && i < pc.n); ++i, ++tile) {      // (a vote: the compiler sees a uniform loop)
                const uint32_t st = tile & 1u, ph = (tile >> 1) & 1u;
                const uint32_t d = tmem_base + kColS + st * 64;
                const uint32_t full = bar_slot_full + 8 * kSlots * st;
                const uint64_t k_desc = umma_smem_desc_sw128(smem_u32(stage_smem + st * kStageBytes));
                // the softmax has read the scores that this buffer held
                ok = wait_warp(bar_s_free + 8 * st, ph ^ 1u) && wait_warp(full + 8 * 4, ph);
                if (!ok) break;
                tcgen05_fence_after_sync();
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) {                                         // the positional block first
                    const uint64_t a_desc = q_desc + 8 * (kRows * 128 / 16) + ks * 2, b_desc = k_desc + 8 * (kBlockBytes / 16) + ks * 2;
                    if (ks) umma_f16_elect<true>(d, a_desc, b_desc, kIdescS);
                    else umma_f16_elect<false>(d, a_desc, b_desc, kIdescS);
                }
                umma_commit_elect(bar_slot_empty + 8 * (kSlots * st + 4));
                uint64_t a_desc = q_desc, b_desc = k_desc;
#pragma unroll 1
                for (int sl = 0; sl < 4; ++sl) {                                         // rolled: the roles share an instruction cache
                    ok = wait_warp(full + 8 * sl, ph);
                    if (!ok) break;
                    tcgen05_fence_after_sync();
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks)
                            umma_f16_elect<true>(d, a_desc + b * (kRows * 128 / 16) + ks * 2, b_desc + b * (kBlockBytes / 16) + ks * 2, kIdescS);
                    a_desc += 2 * (kRows * 128 / 16);
                    b_desc += 2 * (kBlockBytes / 16);
                }
                if (!ok) break;
                umma_commit_elect(bar_s_full + 8 * st);
            }
            if (ok) umma_commit_elect(bar_q_empty);
            ++item;
        }
        if (!ok && lane == 0) give_up(DEV_TIMEOUT_MMA);
    } else if (warp == 1) {
        // ------------------------------------------------------------ P V (a warp of its own: its waits do not hold up the scores)
        constexpr uint32_t kIdescPV = umma_idesc(1, 1, kRows, 128) | kUmmaBMajorMN;
        const uint64_t p_desc = umma_smem_desc_sw128(smem_u32(p_smem));
        while (ok && walk.next(pc)) {
            rows_of(pc.unit, seq, r0);
            ok = wait_warp(bar_o_free, (item & 1u) ^ 1u);                // the previous piece's output has been read
            for (int i = 0; __all_sync(0xFFFFFFFFu, ok && i < pc.n); ++i, ++tile) {
                const uint32_t st = tile & 1u;
                uint64_t v_desc = umma_smem_desc_sw128_mn(smem_u32(stage_smem + st * kStageBytes), kBlockBytes);
                ok = wait_warp(bar_p_ready, tile & 1u);
                if (!ok) break;
                tcgen05_fence_after_sync();
#pragma unroll 1
                for (int sl = 0; sl < 4; ++sl) {                         // 128 value columns: half sl / 2 of O, columns 128 (sl % 2) ..
                    const uint32_t d = tmem_base + (sl & 1) * 128 + (static_cast<uint32_t>((sl >> 1) * 16) << 16);
#pragma unroll
                    for (int ks = 0; ks < kTile / 16; ++ks)
                        umma_f16_elect_acc(d, p_desc + ks * 2, v_desc + ks * (16 * 128 / 16), kIdescPV, (i | ks) ? 1u : 0u);
                    umma_commit_elect(bar_slot_empty + 8 * (kSlots * st + sl));
                    v_desc += 2 * kBlockBytes / 16;
                }
                umma_commit_elect(bar_pv_done);
            }
            ++item;
        }
        if (!ok && lane == 0) give_up(DEV_TIMEOUT_MMA);
    } else if (warp == 2) {
        // ------------------------------------------------------------ Q
        if (lane == 0) {
            int before = 0;                                  // tiles of the piece before
            while (ok && walk.next(pc)) {
                rows_of(pc.unit, seq, r0);
                ok = mbar_wait(bar_q_empty, (item & 1u) ^ 1u, abort_flag, piece_budget(before), 200);
                before = pc.n;
                if (!ok) break;
                mbar_arrive_expect_tx(bar_q_full, kQBytes);
                for (int b = 0; b < kBlocks; ++b)
                    tma_load_2d(smem_u32(q_smem + b * kRows * 128), &q_map, bar_q_full, b * 64, static_cast<int>(seq * seq_rows + r0));
                ++item;
            }
            if (!ok) give_up(DEV_TIMEOUT_PRODUCER);
        }
    } else if (!Q4 && warp == 3) {
        // ------------------------------------------------------------ bf16 rows
        uint32_t tails = 0;
        while (ok && walk.next(pc)) {
            rows_of(pc.unit, seq, r0);
            const int64_t len = seq_len(seq);
            const int64_t base = first_row(p.a, seq);
            for (int i = 0; i < pc.n && ok; ++i, ++tile) {
                const uint32_t st = tile & 1u, ph = ((tile >> 1) & 1u) ^ 1u;
                uint8_t* dst = stage_smem + st * kStageBytes;
                const int64_t at = static_cast<int64_t>(pc.t0 + i) * kTile;
                // coordinates outside the cache read zeros; a base far outside is brought to the nearest such place
                const int64_t first = min(max(base + at, static_cast<int64_t>(-kTile)), p.a.n_kv);
                const bool tail = len - at < kTile;
                // ask the L2 for the tile after the next
                const int64_t soon = base + at + 2 * kTile;
                if (lane == 0 && i + 2 < pc.n && soon >= 0 && soon + kTile <= p.a.n_kv)
                    l2_prefetch(static_cast<const uint8_t*>(p.a.kv) + soon * kLatentBf16RowBytes, kTile * kLatentBf16RowBytes);
                if (!tail) {
#pragma unroll
                    for (int n = 0; n < kSlots; ++n) {
                        const int sl = n == 0 ? 4 : n - 1;           // the order in which the scores take them
                        const uint32_t full = bar_slot_full + 8 * (kSlots * st + sl), to = smem_u32(dst + 2 * sl * kBlockBytes);
                        ok = ok && wait_warp(bar_slot_empty + 8 * (kSlots * st + sl), ph);
                        if (ok && lane == 0) {
                            mbar_arrive_expect_tx(full, (sl == 4 ? 1 : 2) * kBlockBytes);
                            if (sl == 4) tma_load_2d(to, &rope_map, full, 512, static_cast<int>(first));
                            else tma_load_3d(to, &v_map, full, 0, static_cast<int>(first), 2 * sl);
                        }
                    }
                    if (!ok) break;
                } else {
                    // the sequence ends inside this tile: load, clear the rows behind its end, publish
                    for (int sl = 0; sl < kSlots && ok; ++sl) ok = wait_warp(bar_slot_empty + 8 * (kSlots * st + sl), ph, 20);
                    if (!ok) break;
                    if (lane == 0) {
                        mbar_arrive_expect_tx(bar_tail, kStageBytes);
                        for (int b = 0; b < kBlocks; ++b)
                            tma_load_2d(smem_u32(dst + b * kBlockBytes), &rope_map, bar_tail, b * 64, static_cast<int>(first));
                    }
                    ok = wait_warp(bar_tail, tails & 1u);
                    if (!ok) break;
                    ++tails;
                    const int valid = static_cast<int>(len - at);
                    for (int b = 0; b < kBlocks; ++b)
                        for (int o = valid * 128 + lane * 16; o < static_cast<int>(kBlockBytes); o += 512)
                            *reinterpret_cast<uint4*>(dst + b * kBlockBytes + o) = make_uint4(0, 0, 0, 0);
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0)
                        for (int sl = 0; sl < kSlots; ++sl) mbar_arrive(bar_slot_full + 8 * (kSlots * st + sl));
                }
            }
            ++item;
        }
        if (!ok && lane == 0) give_up(DEV_TIMEOUT_GATHER);
    } else if (Q4 && warp >= 8) {
        // ------------------------------------------------------------ 4-bit rows
        // Warps 0..3 fill slots 0 and 2 of every tile, warps 4..7 slots 4 (positional columns), 1 and 3: a slot's hand-over (wait, fence,
        // arrive) takes as long as its copying, so two slots are under way at a time. A warp has rows 16w .. 16w + 15: lane =
        // 8 (2 block + half) + rr reads the 16 bytes (one scale group) of half `half` of a slot's block `block` of rows rr and rr + 8, and
        // stores four 16-byte chunks of each; eight consecutive lanes then store to eight different chunk positions (no bank
        // conflicts). Positional columns: lane = 8 row + chunk, four rows a lane. Everything of the next tile is in registers
        // before this tile's slot is free, expanded before the wait for the slot.
        const int w = (warp - 8) & 3, odd = (warp - 8) >> 2;
        const int rr = lane & 7, blk = lane >> 4, half = (lane >> 3) & 1;
        const uint8_t* kv = static_cast<const uint8_t*>(p.a.kv);
        uint4 code[2][2], rope[4];                            // [slot odd or odd + 2][row rr or rr + 8] of the tile being fetched
        uint16_t scale[2][2];
        uint32_t nx_mask = 0;
        int64_t len = 0, base = 0;
        const int32_t* sel = nullptr;
        int64_t src[2];                                       // cache rows of this lane's rows in the tile being fetched, -1: none
        auto locate = [&](int t) {                            // tile t of the piece's sequence
            nx_mask = 0;
#pragma unroll
            for (int it = 0; it < 2; ++it) {
                int64_t r = static_cast<int64_t>(t) * kTile + w * 16 + it * 8 + rr;
                bool use = r < len;
                if (sel != nullptr) {
                    r = use ? __ldg(sel + r) : -1;
                    use = r >= 0;
                }
                r += base;
                src[it] = use && r >= 0 && r < p.a.n_kv ? r : -1;
                nx_mask |= (__ballot_sync(0xFFFFFFFFu, src[it] >= 0) & 255u) << (8 * it);
            }
        };
        auto fetch_codes = [&](int u) {
            const int cc = (2 * u + odd) * 4 + blk * 2 + half;
#pragma unroll
            for (int it = 0; it < 2; ++it) {
                const uint8_t* row = kv + (src[it] < 0 ? 0 : src[it]) * kLatentQ4RowBytes;
                code[u][it] = src[it] < 0 ? make_uint4(0, 0, 0, 0) : __ldg(reinterpret_cast<const uint4*>(row) + cc);
                scale[u][it] = src[it] < 0 ? static_cast<uint16_t>(0) : __ldg(reinterpret_cast<const uint16_t*>(row + kLatentQ4ScaleOff) + cc);
            }
        };
        auto fetch_rope = [&]() {
#pragma unroll
            for (int it = 0; it < 4; ++it) {
                const int64_t s = __shfl_sync(0xFFFFFFFFu, src[it >> 1], (it & 1) * 4 + (lane >> 3));
                rope[it] = s < 0 ? make_uint4(0, 0, 0, 0) : __ldg(reinterpret_cast<const uint4*>(kv + s * kLatentQ4RowBytes + kLatentQ4RopeOff) + (lane & 7));
            }
        };
        // the piece that the fetches are in runs ahead of the one whose tiles are stored
        Walk ahead = walk;
        Piece apc{};
        int ai = 0;
        bool more = false;
        auto ahead_piece = [&]() {
            more = false;
            if (ahead.next(apc)) {
                const int64_t s = p.tiles.seq_of(apc.unit);
                len = seq_len(s);
                base = first_row(p.a, s);
                sel = p.a.topk ? p.a.topk + s * p.a.k_top : nullptr;
                ai = 0;
                more = true;
            }
        };
        ahead_piece();
        if (more) {
            locate(apc.t0);
            if (odd) fetch_rope();
            fetch_codes(0);
            fetch_codes(1);
        }
        while (more && ok) {
            // store tile `tile` (in registers), fetching the next as the registers come free
            const uint32_t st = tile & 1u, ph = ((tile >> 1) & 1u) ^ 1u;
            uint8_t* dst = stage_smem + st * kStageBytes;
            const uint32_t mask = nx_mask;
            if (++ai == apc.n) ahead_piece();
            if (more) {
                locate(apc.t0 + ai);
                // dense rows lie one behind the other: ask the L2 for a tile further ahead (one warp)
                const int64_t soon = base + static_cast<int64_t>(apc.t0 + ai + 2) * kTile;
                if (sel == nullptr && warp == 8 && lane == 0 && ai + 2 < apc.n && soon >= 0 && soon + kTile <= p.a.n_kv)
                    l2_prefetch(kv + soon * kLatentQ4RowBytes, kTile * kLatentQ4RowBytes);
            }
            auto publish = [&](int sl) {
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_slot_full + 8 * (kSlots * st + sl));
            };
            if (odd) {
                ok = wait_warp(bar_slot_empty + 8 * (kSlots * st + 4), ph);
                if (!ok) break;
#pragma unroll
                for (int it = 0; it < 4; ++it) {
                    const int r = w * 16 + it * 4 + (lane >> 3);
                    *reinterpret_cast<uint4*>(dst + 8 * kBlockBytes + r * 128 + (((lane & 7) ^ (r & 7)) << 4)) = rope[it];
                }
                publish(4);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int sl = 2 * u + odd;
                uint4 value[2][4];
#pragma unroll
                for (int it = 0; it < 2; ++it) {
                    const Q4Scale s2 = q4_scale_of(scale[u][it]);
                    const uint32_t word[4] = {code[u][it].x, code[u][it].y, code[u][it].z, code[u][it].w};
#pragma unroll
                    for (int v = 0; v < 4; ++v) value[it][v] = dequant8_q4(word[v], s2);
                }
                if (more) {                                   // behind the expansion: it must not wait for loads younger than its own
                    if (u == 0 && odd) fetch_rope();
                    fetch_codes(u);
                }
                ok = wait_warp(bar_slot_empty + 8 * (kSlots * st + sl), ph);
                if (!ok) break;
                uint8_t* row = dst + (2 * sl + blk) * kBlockBytes + (w * 16 + rr) * 128;
#pragma unroll
                for (int it = 0; it < 2; ++it)
#pragma unroll
                    for (int v = 0; v < 4; ++v) *reinterpret_cast<uint4*>(row + it * 1024 + (((half * 4 + v) ^ rr) << 4)) = value[it][v];
                if (sl == 0 && lane == 0) *reinterpret_cast<uint16_t*>(mask_smem + st * 8 + 2 * w) = static_cast<uint16_t>(mask);
                publish(sl);
            }
            ++tile;
        }
        if (!ok && lane == 0) give_up(DEV_TIMEOUT_GATHER);
    } else if (warp >= 4 && warp < 8) {
        // ------------------------------------------------------------ softmax and output
        // A warp has 16 query rows (its TMEM lane quarter). Scores are read as 16 x 256-bit fragments: with g = lane / 4 and
        // j = lane % 4 a thread holds rows g and g + 8, columns 8i + 2j + {0, 1}; a row's maximum takes two shuffles.
        const int quarter = warp & 3, g = lane >> 2, j = lane & 3;
        const uint32_t lane_base = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16);
        const int row0 = quarter * 16 + g;
        // lane l gives the address of row l % 8 of matrix l / 8: rows 0..7 | 8..15 of an even chunk, then of the odd one
        const uint32_t p_addr = smem_u32(p_smem) + (quarter * 16 + ((lane >> 3) & 1) * 8 + (lane & 7)) * 128;
        write_empty_units(p, group, quarter, lane, seq_rows, rows_of);
        while (ok && walk.next(pc)) {
            const int n_rows = rows_of(pc.unit, seq, r0);
            // keys that rows g and g + 8 see (dense): the sequence's length less the new tokens behind the row's own
            const int64_t len = seq_len(seq);
            int sees[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = row0 + 8 * h;
                const int64_t n = p.a.topk ? len : len - (p.a.n_step - 1 - (r0 + r) / p.a.H);
                sees[h] = r < n_rows ? static_cast<int>(max(n, int64_t(0))) : 0;
            }
            const int64_t base = first_row(p.a, seq);
            // rows [lo, hi) of the sequence lie inside the cache
            const int lo = static_cast<int>(min(max(-base, int64_t(0)), int64_t(1) << 30));
            const int hi = static_cast<int>(min(max(p.a.n_kv - base, int64_t(0)), int64_t(1) << 30));
            if (!p.a.topk) {
#pragma unroll
                for (int h = 0; h < 2; ++h) sees[h] = min(sees[h], hi);
            }
            float m_ref[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
            for (int i = 0; i < pc.n && ok; ++i, ++tile) {
                const uint32_t st = tile & 1u;
                ok = wait_warp(bar_s_full + 8 * st, (tile >> 1) & 1u);
                if (!ok) break;
                tcgen05_fence_after_sync();
                uint32_t s[2][16];
                tmem_ld_16x256b_x4(lane_base + kColS + st * 64, s[0]);
                tmem_ld_16x256b_x4(lane_base + kColS + st * 64 + 32, s[1]);
                tmem_ld_wait(s[0]);
                tmem_ld_wait(s[1]);
                tcgen05_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_s_free + 8 * st);
                const int at = (pc.t0 + i) * kTile;
                float x[2][16];                                       // [row][8 column groups x 2], not yet scaled
#pragma unroll
                for (int k = 0; k < 8; ++k)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int e = 0; e < 2; ++e) x[h][2 * k + e] = __uint_as_float(s[k >> 2][4 * (k & 3) + 2 * h + e]);
                if (p.sign != 1.f) {                                  // a negative or zero scale: what is scaled grows with the score
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        x[0][k] *= p.sign;
                        x[1][k] *= p.sign;
                    }
                }
                if (Q4 && p.a.topk) {
                    const uint2 mv = *reinterpret_cast<const uint2*>(mask_smem + st * 8);       // byte k: rows 8k .. 8k + 7
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const uint32_t two = (k < 4 ? mv.x : mv.y) >> ((k & 3) * 8 + 2 * j);
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const bool in = (two >> e) & 1u;
                            x[0][2 * k + e] = in && sees[0] ? x[0][2 * k + e] : -INFINITY;
                            x[1][2 * k + e] = in && sees[1] ? x[1][2 * k + e] : -INFINITY;
                        }
                    }
                } else if (__any_sync(0xFFFFFFFFu, at + kTile > min(sees[0], sees[1]) || at < lo)) {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int k = 0; k < 16; ++k) {
                            const int c = at + 8 * (k >> 1) + 2 * j + (k & 1);
                            if (c >= sees[h] || c < lo) x[h][k] = -INFINITY;
                        }
                }
                float alpha[2];
                bool move = false;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float m4[4];                                      // short chains
#pragma unroll
                    for (int k = 0; k < 4; ++k) m4[k] = fmaxf(fmaxf(x[h][k], x[h][k + 4]), fmaxf(x[h][k + 8], x[h][k + 12]));
                    float mt = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
                    mt = fmaxf(mt, __shfl_xor_sync(0xFFFFFFFFu, mt, 1));
                    mt = fmaxf(mt, __shfl_xor_sync(0xFFFFFFFFu, mt, 2)) * p.scale_log2;
                    alpha[h] = 1.f;
                    if (mt > m_ref[h] + kMoveThreshold) {             // also the first usable score (m_ref = -inf)
                        alpha[h] = m_ref[h] == -INFINITY ? 0.f : exp2_fast(m_ref[h] - mt);
                        m_ref[h] = mt;
                        l[h] *= alpha[h];
                        move = true;
                    }
                }
                uint32_t pk[2][8];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float ref = m_ref[h] == -INFINITY ? 0.f : m_ref[h];
                    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const float p0 = exp2_fast(__fmaf_rn(x[h][2 * k], p.scale_log2, -ref)), p1 = exp2_fast(__fmaf_rn(x[h][2 * k + 1], p.scale_log2, -ref));
                        sum[k & 3] += p0 + p1;
                        pk[h][k] = pack2(p0, p1);
                    }
                    l[h] += (sum[0] + sum[1]) + (sum[2] + sum[3]);
                }
                const bool any_move = __any_sync(0xFFFFFFFFu, move);
                // the previous tile's product has read P (and, for a rescale, written O); the piece's first tile: the product before it was
                // waited for when that piece was written out
                if (i > 0) {
                    ok = wait_warp(bar_pv_done, (tile - 1u) & 1u);
                    if (!ok) break;
                    if (any_move) {
                        tcgen05_fence_after_sync();
                        const float a0 = __shfl_sync(0xFFFFFFFFu, alpha[0], (lane & 7) * 4), a1 = __shfl_sync(0xFFFFFFFFu, alpha[1], (lane & 7) * 4);
                        const float f = (lane & 8) ? a1 : a0;             // lanes 0..15 and 16..31: rows 0..15 of the two halves of O
#pragma unroll 1
                        for (int c = 0; c < 8; ++c) {
                            uint32_t o[32];
                            tmem_ld_32x32b_x32(lane_base + c * 32, o);
                            tmem_ld_wait(o);
#pragma unroll
                            for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                            tmem_st_32x32b_x32(lane_base + c * 32, o);
                        }
                        tmem_st_wait();
                    }
                }
#pragma unroll
                for (int c = 0; c < 4; ++c)                           // chunks 2c, 2c + 1 of rows 0..7 and 8..15: four 8 x 8 matrices
                    stmatrix_x4(p_addr + (((2 * c + (lane >> 4)) ^ (lane & 7)) << 4), pk[0][2 * c], pk[1][2 * c], pk[0][2 * c + 1], pk[1][2 * c + 1]);
                fence_proxy_async_smem();
                tcgen05_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_p_ready);
            }
            if (!ok) break;
            ok = wait_warp(bar_pv_done, (tile - 1u) & 1u);
            if (!ok) break;
            tcgen05_fence_after_sync();
            // ---- this thread's rows' sums, then the output: lane = row (lane & 15) of half lane >> 4 of O
            float inv[2], lse[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                l[h] += __shfl_xor_sync(0xFFFFFFFFu, l[h], 1);
                l[h] += __shfl_xor_sync(0xFFFFFFFFu, l[h], 2);
                inv[h] = l[h] != 0.f ? 1.f / l[h] : 0.f;              // 0: the row saw nothing; a sum that is no number stays none
                lse[h] = l[h] != 0.f ? (m_ref[h] + log2f(l[h])) * 0.6931471805599453f : -INFINITY;
            }
            const float i0 = __shfl_sync(0xFFFFFFFFu, inv[0], (lane & 7) * 4), i1 = __shfl_sync(0xFFFFFFFFu, inv[1], (lane & 7) * 4);
            const float f = (lane & 8) ? i1 : i0;
            const int64_t at_row = seq * seq_rows + r0;
            const int64_t slot = (static_cast<int64_t>(group) * 2 + (pc.t0 == 0 ? 1 : 0)) * kRows;
            // this warp's rows of P, which it alone writes and the last product has read, are where it turns its rows
            const uint32_t stage = smem_u32(p_smem) + quarter * 2048;
#pragma unroll 1
            for (int c = 0; c < 8; ++c) {
                uint32_t o[32];
                tmem_ld_32x32b_x32(lane_base + c * 32, o);
                tmem_ld_wait(o);
                uint4 v[4];
                if (pc.whole) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        v[k] = make_uint4(pack2(__uint_as_float(o[8 * k]) * f, __uint_as_float(o[8 * k + 1]) * f),
                                          pack2(__uint_as_float(o[8 * k + 2]) * f, __uint_as_float(o[8 * k + 3]) * f),
                                          pack2(__uint_as_float(o[8 * k + 4]) * f, __uint_as_float(o[8 * k + 5]) * f),
                                          pack2(__uint_as_float(o[8 * k + 6]) * f, __uint_as_float(o[8 * k + 7]) * f));
                    store_rows(stage, lane, v, [&](int r, int i) -> uint4* {
                        const int row = quarter * 16 + (r & 15);
                        return row < n_rows ? reinterpret_cast<uint4*>(p.out + (at_row + row) * 512 + (r >> 4) * 256 + c * 32) + i : nullptr;
                    });
                } else {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            v[k] = make_uint4(__float_as_uint(__uint_as_float(o[16 * e + 4 * k]) * f), __float_as_uint(__uint_as_float(o[16 * e + 4 * k + 1]) * f),
                                              __float_as_uint(__uint_as_float(o[16 * e + 4 * k + 2]) * f), __float_as_uint(__uint_as_float(o[16 * e + 4 * k + 3]) * f));
                        store_rows(stage, lane, v, [&](int r, int i) -> uint4* {
                            const int row = quarter * 16 + (r & 15);
                            return row < n_rows ? reinterpret_cast<uint4*>(p.part_out + (slot + row) * 512 + (r >> 4) * 256 + c * 32 + e * 16) + i : nullptr;
                        });
                    }
                }
            }
            tcgen05_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_o_free);
            if (j == 0) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int r = row0 + 8 * h;
                    if (r >= n_rows) continue;
                    if (!pc.whole) p.part_lse[slot + r] = lse[h];
                    else if (p.lse) p.lse[at_row + r] = lse[h];
                }
            }
            ++item;
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
        tmem_dealloc(tmem_base, 512);
    }
}

// ---------------------------------------------------------------- merge
// A unit cut by runs: group g - 1 holds its beginning (slot 1), groups g, g + 1, .. its continuations (slot 0). Block (g, y)
// takes rows 4 (y + k gridDim.y) .. + 3 of the unit that group g is the first to start inside of; 128 threads a row, 4 columns each. As
// many blocks as run at a time where every unit needs them. Bound by latency and by what is in flight: 32 queries of 32 tiles (the whole call) 44.9 us,
// 64 sequences of 1 to 9 thousand rows 92.3 us; with eight pieces at a time 47.6 and 94.9, with three CTAs of four pieces 44.7 and 94.2, with a
// block for every four rows 2 us more.
constexpr int kMergePieces = 6, kMergeCtas = 2;
__global__ void __launch_bounds__(512, kMergeCtas)
latent_merge_kernel(const Params p) {
    wait_for_previous();
    const int g = blockIdx.x;
    const int2 s = p.starts[g];
    const int run = p.runs[g], run_end = p.runs[g + 1];
    int first = g > 0 ? g - 1 : 0, first_run = p.runs[first];
    int2 fs = p.starts[first];
    if (run_end == run || s.y == 0) return;                   // no tiles, or begins with its unit
    // the run that holds the tile before this one: the nearest earlier non-empty one
    for (int next = run; first > 0 && first_run == next;) {
        next = first_run;
        first_run = p.runs[--first];
        fs = p.starts[first];
    }
    if (fs.x == s.x && fs.y > 0) return;                      // an earlier group starts inside this unit too
    const int end = run - s.y + p.tiles(static_cast<uint32_t>(s.x));      // one past the unit's last tile, end to end
    const uint32_t seq = p.tiles.seq_of(static_cast<uint32_t>(s.x));
    const int seq_rows = p.a.n_step * p.a.H, first_row = static_cast<int>(s.x - seq * p.blocks_per_seq) * p.ways * kRows;
    const int n_rows = min(p.ways * kRows, seq_rows - first_row), c = threadIdx.x & 127;
    const int64_t stride = static_cast<int64_t>(2) * p.ways * kRows;            // rows of a group's two slots
    for (int r = blockIdx.y * 4 + (threadIdx.x >> 7); r < n_rows; r += gridDim.y * 4) {
        const int64_t at1 = first * stride + p.ways * kRows + r, at0 = g * stride + r;
        float m = -INFINITY, z = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        // piece 0 is the beginning, piece k > 0 group g + k - 1's; kMergePieces at a time, all their loads before their first use
        bool more = true;
        for (int k0 = 0; more; k0 += kMergePieces) {
            float ls[kMergePieces];
            float4 v[kMergePieces];
#pragma unroll
            for (int j = 0; j < kMergePieces; ++j) {
                const int k = k0 + j, grp = g + k - 1;
                bool in = k == 0;
                if (k > 0) {
                    const int b0 = grp < p.groups ? p.runs[grp] : end;
                    more = b0 < end;
                    in = more && p.runs[grp + 1] > b0;
                }
                const int64_t at = k == 0 ? at1 : at0 + (k - 1) * stride;
                ls[j] = in ? p.part_lse[at] : -INFINITY;
                v[j] = in ? reinterpret_cast<const float4*>(p.part_out + at * 512)[c] : make_float4(0.f, 0.f, 0.f, 0.f);
            }
            float top = m;
            bool none = m == -INFINITY;                       // (fmaxf passes over what is no number; the weights do not)
#pragma unroll
            for (int j = 0; j < kMergePieces; ++j) {
                top = fmaxf(top, ls[j]);
                none = none && ls[j] == -INFINITY;
            }
            if (none) continue;
            if (top == -INFINITY) top = 0.f;
            const float f = exp2_fast((m - top) * 1.4426950408889634f);
            m = top;
            z *= f;
            acc.x *= f; acc.y *= f; acc.z *= f; acc.w *= f;
#pragma unroll
            for (int j = 0; j < kMergePieces; ++j) {
                const float w = exp2_fast((ls[j] - top) * 1.4426950408889634f);
                acc.x += w * v[j].x; acc.y += w * v[j].y; acc.z += w * v[j].z; acc.w += w * v[j].w;
                z += w;
            }
        }
        const float inv = z != 0.f ? 1.f / z : 0.f;
        const int64_t out_row = static_cast<int64_t>(seq) * seq_rows + first_row + r;
        reinterpret_cast<uint2*>(p.out + out_row * 512)[c] = make_uint2(pack2(acc.x * inv, acc.y * inv), pack2(acc.z * inv, acc.w * inv));
        if (p.lse && c == 0) p.lse[out_row] = z != 0.f ? m + logf(z) : -INFINITY;
    }
}

}  // namespace

int latent_attn_ways(int n_step, int H) { return static_cast<int64_t>(n_step) * H > kRows ? 2 : 1; }

namespace {

struct Layout {
    int ways, blocks_per_seq, groups;
    int64_t units;
    size_t tiles_off, starts_off, runs_off, lse_off, out_off, bytes;
};

Layout layout_of(int64_t B, int n_step, int64_t max_len, int H, int sm_count) {
    Layout y{};
    const int64_t rows = static_cast<int64_t>(n_step) * H;
    y.ways = latent_attn_ways(n_step, H);
    y.blocks_per_seq = static_cast<int>((rows + y.ways * kRows - 1) / (y.ways * kRows));
    y.units = B * y.blocks_per_seq;
    const int64_t most = y.units * ((max_len + kTile - 1) / kTile);
    const int64_t cap = sm_count / y.ways;
    y.groups = static_cast<int>(most < 1 ? 1 : (most < cap ? most : cap));
    auto take = [&](size_t bytes) { const size_t at = y.bytes; y.bytes += (bytes + 255) / 256 * 256; return at; };
    y.tiles_off = take(static_cast<size_t>(B) * 4);            // counted tiles (selected rows)
    y.starts_off = take(static_cast<size_t>(y.groups + 1) * 8);
    y.runs_off = take(static_cast<size_t>(y.groups + 1) * 4);
    const size_t slots = static_cast<size_t>(y.groups) * 2 * y.ways * kRows;
    y.lse_off = take(slots * 4);
    y.out_off = take(slots * 512 * 4);
    return y;
}

}  // namespace

size_t latent_attn_workspace_bytes(int64_t B, int n_step, int64_t max_len, int H) {
    return layout_of(B, n_step, max_len, H, kLatentMaxGrid).bytes;
}

bool latent_attn_fits(int64_t B, int n_step, int64_t max_len, int H) {
    const Layout y = layout_of(B, n_step, max_len, H, kLatentMaxGrid);
    const int64_t tiles = (max_len + kTile - 1) / kTile;
    return y.units < (int64_t(1) << 31) && (tiles == 0 || y.units <= ((int64_t(1) << 31) - 1) / tiles);
}

cudaError_t launch_latent_attn(const LatentArgs& a, void* out, float* lse, void* workspace, const LatentMaps& maps, unsigned int* status, int sm_count,
                               cudaStream_t stream, int* launches) {
    const Layout y = layout_of(a.B, a.n_step, a.max_len, a.H, sm_count < kLatentMaxGrid ? sm_count : kLatentMaxGrid);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    int32_t* tiles = reinterpret_cast<int32_t*>(ws + y.tiles_off);
    int2* starts = reinterpret_cast<int2*>(ws + y.starts_off);
    int32_t* runs = reinterpret_cast<int32_t*>(ws + y.runs_off);
    const UnitTiles unit_tiles{a.topk ? tiles : nullptr, a.lens, a.max_len, static_cast<uint32_t>(y.blocks_per_seq), 6};
    const Params p{a, unit_tiles, starts, runs, static_cast<uint32_t>(y.units), y.blocks_per_seq, y.ways, y.groups, a.scale == 0.f ? 1.f : fabsf(a.scale) * 1.4426950408889634f,
                   a.scale > 0.f ? 1.f : (a.scale < 0.f ? -1.f : 0.f), static_cast<__nv_bfloat16*>(out), lse,
                   reinterpret_cast<float*>(ws + y.out_off), reinterpret_cast<float*>(ws + y.lse_off), status};
    cudaError_t e;
    if (a.topk) {
        ++*launches;
        latent_count_kernel<<<static_cast<unsigned>(a.B), kCountThreads, 0, stream>>>(a, tiles);
        if ((e = cudaGetLastError()) != cudaSuccess) return e;
    }
    ++*launches;
    if (y.ways == 2) {
        e = launch_latent_attn_pair(maps, p, stream);
    } else {
        const void* k = a.q4 ? reinterpret_cast<const void*>(latent_attn_kernel<true>) : reinterpret_cast<const void*>(latent_attn_kernel<false>);
        if ((e = ensure_max_dynamic_smem(k, kSmemBytes)) != cudaSuccess) return e;
        if (a.topk) e = launch_behind(latent_attn_kernel<true>, y.groups, kWarpsQ4 * 32, kSmemBytes, stream, maps.q, maps.rope, maps.v, p);
        else if (a.q4) latent_attn_kernel<true><<<y.groups, kWarpsQ4 * 32, kSmemBytes, stream>>>(maps.q, maps.rope, maps.v, p);
        else latent_attn_kernel<false><<<y.groups, kWarpsBf16 * 32, kSmemBytes, stream>>>(maps.q, maps.rope, maps.v, p);
        if (!a.topk) e = cudaGetLastError();
    }
    if (e != cudaSuccess) return e;
    if (y.groups > 1) {
        ++*launches;
        const int unit_rows = a.n_step * a.H < y.ways * kRows ? a.n_step * a.H : y.ways * kRows;
        const int64_t busy = y.units < y.groups ? y.units : y.groups;          // groups that may have a unit to merge
        const int64_t at_once = kMergeCtas * sm_count / busy, blocks = (unit_rows + 3) / 4;
        e = launch_behind(latent_merge_kernel, dim3(static_cast<unsigned>(y.groups), static_cast<unsigned>(blocks < at_once ? blocks : at_once)), 512, 0, stream, p);
    }
    return e;
}

}  // namespace idxc
