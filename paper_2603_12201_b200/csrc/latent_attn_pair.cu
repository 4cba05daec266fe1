// Attention over latent cache rows for 65 to 128 query rows (all heads of a latent-attention model): a CTA pair on one tile.
//
// tcgen05.mma.cta_group::2 with M = 128 gives each CTA of the pair 64 query rows and issues at the full rate, where two CTAs with
// M = 64 of their own issue at half of it (measured: N = 64 in 29 clocks, N = 256 in 64, against 32 and 128 for half the rows). Its
// accumulator puts the first half of the N columns on TMEM lanes 0..63 and the second on lanes 64..127, so a CTA holds
//   S: 32 columns, lane r = (row r, first 32 cache rows of the tile), lane 64 + r = (row r, last 32)
//   O: 256 columns, lane r = (row r, value columns 0..255), lane 64 + r = (row r, value columns 256..511)
// and 64 rows x 512 columns of fp32 output are half of tensor memory.
// The B operand is split by columns of the product: for the scores CTA c holds the 576 columns of cache rows 32c .. 32c + 31 (K),
// for P V the value columns 256c .. 256c + 255 of all 64 rows (V). The two overlap, but lie at the same shared-memory offset in both
// CTAs, so they are two buffers, each double-buffered: K is free when the scores are done, V when the product is, and neither
// waits for the other's tile. (One shared buffer a tile, as for up to 64 rows, refills only after the product: 2.8 K clocks a tile.)
// The first CTA's warps 0 and 1 issue for both; loaders and softmax warps of both CTAs arrive on the first one's barriers, and
// commits are multicast to both.
// Shared memory of a CTA: Q 9 x [64 x 128 B] | K 2 x 9 x [32 x 128 B] | V 2 x 4 x [64 x 128 B] | P 2 x [64 x 128 B]. What MMAs read, copies
// write and loads bring passes the same path at 128 bytes a clock, and that path bounds the kernel (selected 4-bit rows: 2800 of its
// wavefronts in 2680 clocks a tile, a load taking one for every 32 bytes). So 6 of Q's 9 blocks are the A operand from tensor memory, in both
// lane halves (each multiplies its own half of the N columns): 384 wavefronts a tile less, selected rows (2047 queries of 2048) 1.18 ->
// 1.13 ms, bf16 rows (32 x 16K to 64K) 378 -> 369 us.
// 4-bit rows in order are copied as they are into a ring of half tiles (3 x 32 rows x 416 B, a bulk copy each), and eight warps expand
// them into K and V; the ring lies where Q's 6 blocks would, so the softmax warps bring those from global to tensor memory themselves: 325 us
// at 8 x 131072 rows, 342 with the rows read straight into registers and Q in shared memory. Selected rows are read straight into
// registers: through the ring 2.1 ms (a copy a row, or 16 bytes at a time: the ring is too short for their latency).
#include <type_traits>

#include "latent_attn.cuh"

namespace idxc {
using namespace latent;
namespace {

constexpr int kHalf = kTile / 2;                    // cache rows of a CTA's K
constexpr uint32_t kKBlock = kHalf * 128;
constexpr uint32_t kKBytes = kBlocks * kKBlock;
constexpr uint32_t kVBlock = kTile * 128;
constexpr uint32_t kVBytes = 4 * kVBlock;
constexpr uint32_t kPBytes = kRows * 128;
constexpr uint32_t kBarBytes = 512;
constexpr uint32_t kSwapBytes = 3 * 4 * 32 * 4;     // what two warps exchange: row maxima, double-buffered, and at the end row sums
constexpr int kQT = 6;                              // Q blocks that the scores take from tensor memory
constexpr int kCopyTiles = 4;                       // they are copied there for pieces of that many tiles (860 clocks; one tile a piece: 0.5 us more)
constexpr int kRawSlots = 3;
constexpr int kCutTiles = 13;                       // (see find_run) selected rows, 50 queries of 32 tiles: 64 us cut even, 58 us apart; 38 of 16: 41 us and 36
constexpr uint32_t kRawBytes = kHalf * kLatentQ4RowBytes;
enum Rows { kBf16, kCodes, kPicked };               // bf16 rows in order, 4-bit rows in order, selected 4-bit rows
constexpr uint32_t q_bytes(Rows r) { return (r == kCodes ? kBlocks - kQT : kBlocks) * kRows * 128; }
constexpr uint32_t smem_bytes(Rows r) {
    return q_bytes(r) + 2 * kKBytes + 2 * kVBytes + 2 * kPBytes + (r == kCodes ? kRawSlots * kRawBytes : 0) + kBarBytes + kSwapBytes + 1024;
}
static_assert(smem_bytes(kBf16) <= 232448 && smem_bytes(kCodes) <= 232448 && smem_bytes(kPicked) <= 232448, "shared memory of a CTA");
constexpr uint32_t kColS = 256;                     // S buffer b at kColS + 32 b; O in [0, 256)
constexpr uint32_t kColQ = 320;                     // Q blocks 0 .. kQT - 1, 32 columns each (two bf16 a column)
constexpr int kWarpsBf16 = 9;                       // 0 scores | 1 P V | 2 Q | 3 K (TMA) | 4..7 softmax | 8 V (TMA)
constexpr int kWarpsQ4 = 16;                        // 0 scores | 1 P V | 2 Q | 3 rows in order | 4..7 softmax | 8..11 K | 12..15 V

// barrier over the two warps of 64 threads that share query rows; returns whether both came with ok
__device__ __forceinline__ bool pair_of_warps_ok(int id, bool ok) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %2, 0;\n\t"
        "barrier.cta.red.and.pred p, %1, 64, q;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(r) : "r"(id), "r"(static_cast<uint32_t>(ok)) : "memory");
    return r != 0;
}

template <Rows ROWS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__((ROWS == kBf16 ? kWarpsBf16 : kWarpsQ4) * 32, 1)
latent_attn_pair_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
                        const __grid_constant__ CUtensorMap rope_map, const __grid_constant__ CUtensorMap v_map, const Params p) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint8_t* q_smem = smem;
    uint8_t* k_smem = q_smem + q_bytes(ROWS);
    uint8_t* v_smem = k_smem + 2 * kKBytes;
    uint8_t* p_smem = v_smem + 2 * kVBytes;
    uint64_t* bars = reinterpret_cast<uint64_t*>(p_smem + 2 * kPBytes);
    uint8_t* raw_smem = p_smem + 2 * kPBytes + kBarBytes + kSwapBytes;
    float* swap = reinterpret_cast<float*>(p_smem + 2 * kPBytes + kBarBytes);        // [3][4 warps][32]
    // barriers that the first CTA's issuing warps wait on (both CTAs arrive there)
    const uint32_t bar_q_full = smem_u32(bars + 0);
    const uint32_t bar_k_full = smem_u32(bars + 1);          // [2]
    const uint32_t bar_v_full = smem_u32(bars + 3);          // [2]
    const uint32_t bar_s_free = smem_u32(bars + 5);          // [2]
    const uint32_t bar_p_ready = smem_u32(bars + 7);         // [2]
    const uint32_t bar_o_free = smem_u32(bars + 9);
    // barriers that commits reach in both CTAs
    const uint32_t bar_q_empty = smem_u32(bars + 10);
    const uint32_t bar_s_full = smem_u32(bars + 11);         // [2] the scores of a tile are done (and its K is free)
    const uint32_t bar_pv_done = smem_u32(bars + 13);        // [2] the product of a tile is done (and its V and P are free)
    const uint32_t bar_tail = smem_u32(bars + 15);
    uint32_t* tmem_base_slot = reinterpret_cast<uint32_t*>(bars + 16);
    volatile uint32_t* abort_flag = tmem_base_slot + 1;
    // 4-bit rows: half tiles that have landed, and that were read; Q's first blocks are in tensor memory
    const uint32_t bar_raw_full = smem_u32(bars + 18);       // [3]
    const uint32_t bar_raw_empty = smem_u32(bars + 21);      // [3]
    const uint32_t bar_q_ready = smem_u32(bars + 24);
    volatile uint8_t* raw_mask = reinterpret_cast<volatile uint8_t*>(bars + 25);         // [3][8] usable rows of a half tile in the ring, four to a byte
    // selected rows: [4 tiles][2 halves][4] usable rows of a tile, eight to a byte. Four deep: K of tile i + 2 may land before the softmax has
    // looked at tile i, but that of tile i + 4 follows the scores of tile i + 2, which waited for the softmax of tile i.
    volatile uint8_t* mask_smem = reinterpret_cast<volatile uint8_t*>(bars + 28);
    static_assert(32 * 8 <= kBarBytes, "barrier area");

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = static_cast<int>(cluster_ctarank());
    const int group = blockIdx.x >> 1;
    const int seq_rows = p.a.n_step * p.a.H;
    auto rows_of = [&](uint32_t unit, int64_t& seq, int& r0) -> int {
        const uint32_t s = p.tiles.seq_of(unit);
        seq = s;
        r0 = (static_cast<int>(unit - s * p.blocks_per_seq) * 2 + rank) * kRows;
        return min(kRows, seq_rows - r0);
    };
    auto seq_len = [&](int64_t seq) -> int64_t {
        return p.a.topk ? p.a.k_top : min(max(static_cast<int64_t>(__ldg(p.a.lens + seq)), int64_t(0)), p.a.max_len);
    };
    auto in_first = [&](uint32_t bar) -> uint32_t { return map_to_cta(bar, 0); };

    let_next_start();                                        // the merge
    EarlyTiles early{};
    if (ROWS != kPicked) early = early_tiles(p.units, p.tiles);
    early_bases(p.a.kv_base, p.a.B);
    if (lane == 0 && warp == 2) tma_prefetch_desc(&q_map);
    if (ROWS == kBf16 && lane == 0 && warp == 3) {
        tma_prefetch_desc(&k_map);
        tma_prefetch_desc(&rope_map);
    }
    if (ROWS == kBf16 && lane == 0 && warp == 8) tma_prefetch_desc(&v_map);
    if (threadIdx.x == 0) {
        mbar_init(bar_q_full, 2);
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar_k_full + 8 * i, ROWS == kBf16 ? 2 : 8);
            mbar_init(bar_v_full + 8 * i, ROWS == kBf16 ? 2 : 8);
            mbar_init(bar_s_free + 8 * i, 8);
            mbar_init(bar_p_ready + 8 * i, 8);
            mbar_init(bar_s_full + 8 * i, 1);
            mbar_init(bar_pv_done + 8 * i, 1);
        }
        mbar_init(bar_o_free, 8);
        mbar_init(bar_q_empty, 1);
        mbar_init(bar_tail, 1);
        mbar_init(bar_q_ready, 8);
        for (int i = 0; i < kRawSlots; ++i) {
            mbar_init(bar_raw_full + 8 * i, 1);
            mbar_init(bar_raw_empty + 8 * i, 8);
        }
        *abort_flag = 0u;
        fence_mbar_init();
    }
    if (warp == 0) {
        tmem_alloc_pair(smem_u32(tmem_base_slot), 512);
        tmem_relinquish_pair();
    }
    tcgen05_fence_before_sync();
    __syncwarp();
    cluster_arrive();                                        // the other CTA's barriers are waited for below
    if (ROWS == kPicked) {                                   // (counted by the kernel before)
        wait_for_previous();
        early = early_tiles(p.units, p.tiles);
    }
    const Run run = find_run(p.units, p.tiles, early, group, p.groups, kCutTiles, reinterpret_cast<int*>(q_smem));      // (Q has not been asked for yet)
    if (threadIdx.x == 0 && rank == 0) {
        p.starts[group] = make_int2(static_cast<int>(run.unit), run.t);
        p.runs[group] = run.first;
        if (group == p.groups - 1) p.runs[p.groups] = run.total;
    }
    fence_proxy_async_smem();                                // find_run's words before Q's copy over them
    if (p.units > kFewUnits) __syncthreads();
    cluster_wait();
    tcgen05_fence_after_sync();
    const uint32_t tmem_base = *tmem_base_slot;

    Walk walk(p.tiles, run);
    Piece pc{};
    int64_t seq;
    int r0;
    bool ok = true;
    uint32_t tile = 0, item = 0;          // counted over the whole kernel: buffers and phases follow from them
    auto give_up = [&](unsigned int code) {
        *abort_flag = 1u;
        st_cluster_u32(map_to_cta(smem_u32(const_cast<uint32_t*>(abort_flag)), static_cast<uint32_t>(rank ^ 1)), 1u);
        atomicCAS(p.status, 0u, code);
    };
    auto wait_warp = [&](uint32_t bar, uint32_t parity) -> bool { return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, abort_flag)); };

    if (warp == 0) {
        // ------------------------------------------------------------ scores (first CTA, warp-uniform)
        constexpr uint32_t kIdescS = umma_idesc(1, 1, 128, kTile);
        const uint64_t q_desc = umma_smem_desc_sw128(smem_u32(q_smem));
        while (rank == 0 && ok && walk.next(pc)) {
            ok = wait_warp(bar_q_full, item & 1u) && (ROWS != kCodes || wait_warp(bar_q_ready, item & 1u));
            const bool in_tmem = ROWS == kCodes || __all_sync(0xFFFFFFFFu, pc.n >= kCopyTiles);      // (a vote: uniform to the compiler)
            if (ROWS != kCodes && __all_sync(0xFFFFFFFFu, ok && in_tmem)) {      // (Q came after the scores that read the last one were done)
                tcgen05_fence_after_sync();
#pragma unroll 1
                for (int b = 0; b < kQT; ++b) tmem_copy_64x128_pair(tmem_base + kColQ + b * 32, q_desc + b * (kRows * 128 / 16));
            }
            for (int i = 0; __all_sync(0xFFFFFFFFu, ok && i < pc.n); ++i, ++tile) {      // (a vote: the compiler sees a uniform loop)
                const uint32_t st = tile & 1u, ph = (tile >> 1) & 1u;
                ok = wait_warp(bar_s_free + 8 * st, ph ^ 1u) && wait_warp(bar_k_full + 8 * st, ph);
                if (!ok) break;
                tcgen05_fence_after_sync();
                const uint32_t d = tmem_base + kColS + st * 32;
                uint64_t b_desc = umma_smem_desc_sw128(smem_u32(k_smem + st * kKBytes));
                auto from_smem = [&](uint64_t a_desc, auto first) {      // blocks first .. 8 of Q
#pragma unroll 3
                    for (int b = first; b < kBlocks; ++b) {
                        umma_f16_pair_x4<2, 2>(d, a_desc, b_desc, kIdescS, b != 0 ? 1u : 0u);
                        a_desc += kRows * 128 / 16;
                        b_desc += kKBlock / 16;
                    }
                };
                if (in_tmem) {
                    uint32_t a_tmem = tmem_base + kColQ;
#pragma unroll 3
                    for (int b = 0; b < kQT; ++b) {
                        umma_f16_pair_ts_x4<2>(d, a_tmem, b_desc, kIdescS, b != 0 ? 1u : 0u);
                        a_tmem += 32;
                        b_desc += kKBlock / 16;
                    }
                    from_smem(q_desc + (ROWS == kCodes ? 0 : kQT * (kRows * 128 / 16)), std::integral_constant<int, kQT>());
                } else {
                    from_smem(q_desc, std::integral_constant<int, 0>());
                }
                umma_commit_pair_elect(bar_s_full + 8 * st);
            }
            if (ok) umma_commit_pair_elect(bar_q_empty);
            ++item;
        }
        if (!ok && lane == 0) give_up(DEV_TIMEOUT_MMA);
    } else if (warp == 1) {
        // ------------------------------------------------------------ P V (first CTA)
        constexpr uint32_t kIdescPV = umma_idesc(1, 1, 128, 256) | kUmmaBMajorMN;
        while (rank == 0 && ok && walk.next(pc)) {
            ok = wait_warp(bar_o_free, (item & 1u) ^ 1u);                // the previous piece's output has been read
            for (int i = 0; __all_sync(0xFFFFFFFFu, ok && i < pc.n); ++i, ++tile) {
                const uint32_t st = tile & 1u, ph = (tile >> 1) & 1u;
                ok = wait_warp(bar_v_full + 8 * st, ph) && wait_warp(bar_p_ready + 8 * st, ph);
                if (!ok) break;
                tcgen05_fence_after_sync();
                const uint64_t p_desc = umma_smem_desc_sw128(smem_u32(p_smem + st * kPBytes));
                const uint64_t v_desc = umma_smem_desc_sw128_mn(smem_u32(v_smem + st * kVBytes), kVBlock);
#pragma unroll
                for (int h = 0; h < 2; ++h)                              // 128 value columns of each CTA
                    umma_f16_pair_x4<2, 16 * 128 / 16>(tmem_base + h * 128, p_desc, v_desc + h * (2 * kVBlock / 16), kIdescPV, i != 0 ? 1u : 0u);
                umma_commit_pair_elect(bar_pv_done + 8 * st);
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
                const uint32_t full = in_first(bar_q_full);
                mbar_arrive_expect_tx_cluster(full, q_bytes(ROWS));
                constexpr int first = ROWS == kCodes ? kQT : 0;          // (the others go to tensor memory by the softmax warps)
                for (int b = first; b < kBlocks; ++b)
                    tma_load_2d_pair(smem_u32(q_smem + (b - first) * kRows * 128), &q_map, full, b * 64, static_cast<int>(seq * seq_rows + r0));
                ++item;
            }
            if (!ok) give_up(DEV_TIMEOUT_PRODUCER);
        }
    } else if (ROWS == kBf16 && warp == 3) {
        // ------------------------------------------------------------ K, bf16: rows 32 rank .. of every tile. Rows behind the sequence's end
        // may hold anything: they only reach scores that the softmax discards.
        if (lane == 0) {
            while (ok && walk.next(pc)) {
                const int64_t base = first_row(p.a, p.tiles.seq_of(pc.unit));
                for (int i = 0; i < pc.n && ok; ++i, ++tile) {
                    const uint32_t st = tile & 1u;
                    const int64_t at = base + static_cast<int64_t>(pc.t0 + i) * kTile;
                    // ask the L2 for a tile further ahead
                    const int64_t soon = at + 3 * kTile;
                    if (rank == 0 && i + 3 < pc.n && soon >= 0 && soon + kTile <= p.a.n_kv)
                        l2_prefetch(static_cast<const uint8_t*>(p.a.kv) + soon * kLatentBf16RowBytes, kTile * kLatentBf16RowBytes);
                    ok = mbar_wait(bar_s_full + 8 * st, ((tile >> 1) & 1u) ^ 1u, abort_flag);
                    if (!ok) break;
                    const int first = static_cast<int>(min(max(at + rank * kHalf, static_cast<int64_t>(-kHalf)), p.a.n_kv));
                    const uint32_t full = in_first(bar_k_full + 8 * st), to = smem_u32(k_smem + st * kKBytes);
                    mbar_arrive_expect_tx_cluster(full, kKBytes);
                    tma_load_3d_pair(to, &k_map, full, 0, first, 0);
                    tma_load_2d_pair(to + 8 * kKBlock, &rope_map, full, 512, first);
                }
            }
            if (!ok) give_up(DEV_TIMEOUT_GATHER);
        }
    } else if (ROWS == kBf16 && warp == 8) {
        // ------------------------------------------------------------ V, bf16: value columns 256 rank .. of every tile
        uint32_t tails = 0;
        while (ok && walk.next(pc)) {
            rows_of(pc.unit, seq, r0);
            const int64_t len = seq_len(seq);
            const int64_t base = first_row(p.a, seq);
            for (int i = 0; i < pc.n && ok; ++i, ++tile) {
                const uint32_t st = tile & 1u;
                const int64_t at = static_cast<int64_t>(pc.t0 + i) * kTile;
                ok = wait_warp(bar_pv_done + 8 * st, ((tile >> 1) & 1u) ^ 1u);
                if (!ok) break;
                const int first = static_cast<int>(min(max(base + at, static_cast<int64_t>(-kTile)), p.a.n_kv));
                uint8_t* dst = v_smem + st * kVBytes;
                const uint32_t full = in_first(bar_v_full + 8 * st);
                if (len - at >= kTile) {
                    if (lane == 0) {
                        mbar_arrive_expect_tx_cluster(full, kVBytes);
                        tma_load_3d_pair(smem_u32(dst), &v_map, full, 0, first, 4 * rank);
                    }
                } else {
                    // the sequence ends inside this tile: load, clear the rows behind its end (0 x NaN would reach the output), publish
                    if (lane == 0) {
                        mbar_arrive_expect_tx(bar_tail, kVBytes);
                        tma_load_3d(smem_u32(dst), &v_map, bar_tail, 0, first, 4 * rank);
                    }
                    ok = wait_warp(bar_tail, tails & 1u);
                    if (!ok) break;
                    ++tails;
                    const int valid = static_cast<int>(len - at);
                    for (int b = 0; b < 4; ++b)
                        for (int o = valid * 128 + lane * 16; o < static_cast<int>(kVBlock); o += 512)
                            *reinterpret_cast<uint4*>(dst + b * kVBlock + o) = make_uint4(0, 0, 0, 0);
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(full);
                }
            }
        }
        if (!ok && lane == 0) give_up(DEV_TIMEOUT_GATHER);
    } else if (ROWS == kCodes && warp == 3) {
        // ------------------------------------------------------------ 4-bit rows in order into the ring, one copy a half tile: of every tile this
        // CTA's half, then the other
        const uint8_t* kv = static_cast<const uint8_t*>(p.a.kv);
        uint32_t slot = 0, ph = 1;
        while (ok && walk.next(pc)) {
            const int64_t s = p.tiles.seq_of(pc.unit);
            const int len = static_cast<int>(seq_len(s));
            const int64_t base = first_row(p.a, s);
            for (int x = 0; x < 2 * pc.n && ok; ++x) {
                const int at = (pc.t0 + (x >> 1)) * kTile + ((x & 1) ^ rank) * kHalf + lane;
                const int64_t r = base + at;
                const uint32_t valid = __ballot_sync(0xFFFFFFFFu, at < len && r >= 0 && r < p.a.n_kv);
                ok = wait_warp(bar_raw_empty + 8 * slot, ph);
                if (!ok) break;
                const uint32_t full = bar_raw_full + 8 * slot;
                if (lane < 8) raw_mask[slot * 8 + lane] = static_cast<uint8_t>((valid >> (4 * lane)) & 15u);
                __syncwarp();
                if (lane == 0) mbar_arrive_expect_tx(full, __popc(valid) * kLatentQ4RowBytes);
                __syncwarp();
                if (valid != 0 && lane == __ffs(valid) - 1)
                    bulk_load_1d(smem_u32(raw_smem) + slot * kRawBytes + lane * kLatentQ4RowBytes, kv + r * kLatentQ4RowBytes,
                                 __popc(valid) * kLatentQ4RowBytes, full);
                // ask the L2 for a tile further ahead
                const int64_t soon = base + static_cast<int64_t>(pc.t0 + (x >> 1) + 4) * kTile;
                if (lane == 31 && (x & 1) == 0 && rank == 0 && (x >> 1) + 4 < pc.n && soon >= 0 && soon + kTile <= p.a.n_kv)
                    l2_prefetch(kv + soon * kLatentQ4RowBytes, kTile * kLatentQ4RowBytes);
                if (++slot == kRawSlots) {
                    slot = 0;
                    ph ^= 1u;
                }
            }
        }
        if (!ok && lane == 0) give_up(DEV_TIMEOUT_PRODUCER);
    } else if (ROWS == kPicked && warp >= 8) {
        // ------------------------------------------------------------ selected 4-bit rows, read and expanded by four warps for K and four for V
        // Lane = 8 c + rr reads the 32 bytes of codes of 64-column block c (or c + 4) of a row rr and stores them as eight 16-byte pieces;
        // eight consecutive lanes then store to eight different positions of the swizzle (no bank conflicts). K's lanes also move 32 bytes of
        // the positional columns. While a tile is stored the next is in registers or on its way there, and the rows of the one
        // after are looked up (a load takes about 1000 clocks). The code is rolled and shared by the two kinds on purpose: unrolled over
        // the tiles in registers the roles stalled on instruction fetch (3300 clocks a tile).
        const bool is_v = warp >= 12;
        const int w = warp & 3, rr = lane & 7, c4 = lane >> 3;
        const uint8_t* kv = static_cast<const uint8_t*>(p.a.kv);
        // this lane's rows of a tile. K: one of this CTA's half, and (for the mask) the same one of the other half; V: two
        const int off0 = is_v ? w * 16 + rr : rank * kHalf + w * 8 + rr, off1 = is_v ? off0 + 8 : (rank ^ 1) * kHalf + w * 8 + rr;
        struct Share { uint32_t code0[8], code1[8], rope[8], scale0, scale1, mask; } cur, nxt;      // this lane's of a tile
        int64_t base = 0;
        int len = 0, raw0 = -1, raw1 = -1;                    // raw: selected position of this lane's rows in the next tile to fetch
        const int32_t* sel = nullptr;
        int i = 0;
        auto open_piece = [&]() {
            if (!walk.next(pc)) return;
            seq = p.tiles.seq_of(pc.unit);
            len = static_cast<int>(seq_len(seq));
            base = first_row(p.a, seq);
            sel = p.a.topk + seq * p.a.k_top;
            i = 0;
        };
        auto look_up = [&]() {
            const int at = (pc.t0 + i) * kTile;
            raw0 = at + off0 < len ? at + off0 : -1;
            raw1 = at + off1 < len ? at + off1 : -1;
            if (raw0 >= 0) raw0 = __ldg(sel + raw0);
            if (raw1 >= 0) raw1 = __ldg(sel + raw1);
        };
        auto cache_row = [&](int raw) -> int {                // -1: takes no part
            const int64_t r = base + raw;
            return raw >= 0 && r >= 0 && r < p.a.n_kv ? static_cast<int>(r) : -1;
        };
        auto fetch = [&](Share& f) {                          // the tile that was looked up; then looks up the next
            const int s0 = cache_row(raw0);
            int s1 = cache_row(raw1);
            {
                const uint32_t mine = __ballot_sync(0xFFFFFFFFu, s0 >= 0) & 255u, theirs = __ballot_sync(0xFFFFFFFFu, s1 >= 0) & 255u;
                f.mask = rank == 0 ? mine | (theirs << 8) : theirs | (mine << 8);     // K: bits 0..7: in the first half of the tile, 8..15: the second
            }
            s1 = is_v ? s1 : s0;
            const int block0 = is_v ? 4 * rank + c4 : c4, block1 = is_v ? block0 : c4 + 4;
            const uint8_t* row0 = kv + static_cast<uint64_t>(static_cast<uint32_t>(max(s0, 0))) * kLatentQ4RowBytes;
            const uint8_t* row1 = kv + static_cast<uint64_t>(static_cast<uint32_t>(max(s1, 0))) * kLatentQ4RowBytes;
            load_nc_256(row0 + block0 * 32, s0 >= 0, f.code0);
            load_nc_256(row1 + block1 * 32, s1 >= 0, f.code1);
            load_nc_256(row0 + kLatentQ4RopeOff + c4 * 32, s0 >= 0 && !is_v, f.rope);
            f.scale0 = load_nc_32(row0 + kLatentQ4ScaleOff + block0 * 4, s0 >= 0);
            f.scale1 = load_nc_32(row1 + kLatentQ4ScaleOff + block1 * 4, s1 >= 0);
            if (++i == pc.n) open_piece();
            look_up();
        };
        const uint32_t bar_free = is_v ? bar_pv_done : bar_s_full, bar_full = in_first(is_v ? bar_v_full : bar_k_full);
        const uint32_t buf_bytes = is_v ? kVBytes : kKBytes, step = is_v ? 1024u : 4 * kKBlock;       // from the first 64 columns of this lane to the second
        // piece v of a row goes to chunk v ^ rr of its 128 bytes: an exclusive or on the address, whose low seven bits hold rr
        const uint32_t my_dst = (is_v ? smem_u32(v_smem) + c4 * kVBlock + off0 * 128 : smem_u32(k_smem) + c4 * kKBlock + (w * 8 + rr) * 128) + (rr << 4);
        const uint32_t rope_dst = smem_u32(k_smem) + 8 * kKBlock + (w * 8 + rr) * 128 + (((2 * c4) ^ rr) << 4);
        const int total = run.n;
        if (total > 0) {
            open_piece();
            look_up();
            fetch(nxt);
        }
#pragma unroll 1
        for (int t = 0; t < total; ++t) {
            const uint32_t st = t & 1;
            cur = nxt;                                        // (waits for the loads: they were issued a tile ago)
            if (t + 1 < total) fetch(nxt);
            ok = wait_warp(bar_free + 8 * st, ((static_cast<uint32_t>(t) >> 1) & 1u) ^ 1u);
            if (!ok) break;
            uint32_t to = my_dst + st * buf_bytes;
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                const Q4Scale lo = q4_scale_of(cur.scale0), hi = q4_scale_of(cur.scale0 >> 16);
#pragma unroll
                for (int v = 0; v < 8; ++v) st_shared_v4(to ^ (v << 4), dequant8_q4(cur.code0[v], v < 4 ? lo : hi));
#pragma unroll
                for (int v = 0; v < 8; ++v) cur.code0[v] = cur.code1[v];
                cur.scale0 = cur.scale1;
                to += step;
            }
            if (!is_v) {
                st_shared_v4(rope_dst + st * kKBytes, make_uint4(cur.rope[0], cur.rope[1], cur.rope[2], cur.rope[3]));
                st_shared_v4((rope_dst + st * kKBytes) ^ 16u, make_uint4(cur.rope[4], cur.rope[5], cur.rope[6], cur.rope[7]));
                if (lane < 2) mask_smem[((t & 3) * 2 + lane) * 4 + w] = static_cast<uint8_t>(cur.mask >> (8 * lane));
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(bar_full + 8 * st);
        }
        if (!ok && lane == 0) give_up(DEV_TIMEOUT_GATHER);
    } else if (ROWS == kCodes && warp >= 8) {
        // ------------------------------------------------------------ 4-bit rows, expanded by four warps for K and four for V
        // A lane has four pieces of a tile, each the 16 bytes of codes under one scale, which become four 16-byte pieces of operand.
        // lane = 8 g + 2 rr + half: 64-column block g (K: then g + 4; V: 4 rank + g), half `half` of it, row rr of four. Eight consecutive
        // lanes then read 32 bytes of four rows, which lie 416 bytes apart (four different quarters of the banks), and store to eight
        // different positions of the swizzle: neither side has bank conflicts. Pieces t = 0..3: rows 8w + 4 (t % 2) + rr of a half tile; K: all of
        // this CTA's half, V: of its half and of the other. The code is rolled and shared by the two kinds on purpose: unrolled, the roles
        // stalled on instruction fetch.
        const bool is_v = warp >= 12;
        const int w = warp & 3, g = lane >> 3, rr = (lane >> 1) & 3, half = lane & 1;
        const uint32_t raw = smem_u32(raw_smem);
        const uint32_t my_row = w * 8 + rr;                   // t even; t odd: 4 more
        const uint32_t my_chunk = 2 * (is_v ? 4 * rank + g : g) + half;
        const uint32_t bar_free = is_v ? bar_pv_done : bar_s_full, bar_full = in_first(is_v ? bar_v_full : bar_k_full);
        const uint32_t buf_bytes = is_v ? kVBytes : kKBytes;
        // piece v of a 32-column group goes to chunk (4 half + v) ^ (row % 8) of its 128 bytes: exclusive ors on an address whose low
        // seven bits hold (4 half) ^ rr; rows of odd t have bit 2 of the row set
        const uint32_t my_dst = (is_v ? smem_u32(v_smem) + g * kVBlock + rank * kHalf * 128 : smem_u32(k_smem) + g * kKBlock) + my_row * 128 + (((4 * half) ^ rr) << 4);
        const int32_t to_second = is_v ? (rank == 0 ? 1 : -1) * kHalf * 128 : static_cast<int32_t>(4 * kKBlock);      // from t = 0, 1 to t = 2, 3
        const uint32_t rope_src = (w * 8 + (lane >> 3)) * kLatentQ4RowBytes + kLatentQ4RopeOff + (lane & 7) * 16;
        const uint32_t rope_dst = smem_u32(k_smem) + 8 * kKBlock + (w * 8 + (lane >> 3)) * 128 + (((lane & 7) ^ (lane >> 3)) << 4);
        uint32_t slot = 0, raw_ph = 0;
        auto next_slot = [&]() {
            if (++slot == kRawSlots) {
                slot = 0;
                raw_ph ^= 1u;
            }
        };
        auto done_with = [&](uint32_t s) {
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_raw_empty + 8 * s);
        };
        uint4 code[4], rope[2] = {};
        uint32_t scale[4];
        auto read = [&](uint4& c0, uint4& c1, uint32_t& s0, uint32_t& s1, uint32_t chunk) {        // pieces of rows my_row and my_row + 4
            const uint32_t at = raw + slot * kRawBytes + my_row * kLatentQ4RowBytes;
            const uint32_t valid = raw_mask[slot * 8 + 2 * w] >> rr, valid4 = raw_mask[slot * 8 + 2 * w + 1] >> rr;
            c0 = ld_shared_v4(at + chunk * 16);
            c1 = ld_shared_v4(at + 4 * kLatentQ4RowBytes + chunk * 16);
            s0 = (valid & 1u) ? ld_shared_u16(at + kLatentQ4ScaleOff + chunk * 2) : 0u;
            s1 = (valid4 & 1u) ? ld_shared_u16(at + 4 * kLatentQ4RowBytes + kLatentQ4ScaleOff + chunk * 2) : 0u;
        };
        const int total = run.n;
#pragma unroll 1
        for (int t = 0; t < total; ++t) {
            const uint32_t st = t & 1;
            ok = wait_warp(bar_raw_full + 8 * slot, raw_ph);
            if (!ok) break;
            read(code[0], code[1], scale[0], scale[1], my_chunk);
            if (!is_v) {
                read(code[2], code[3], scale[2], scale[3], my_chunk + 8);
                const uint32_t valid = raw_mask[slot * 8 + 2 * w] >> (lane >> 3), valid4 = raw_mask[slot * 8 + 2 * w + 1] >> (lane >> 3);
                rope[0] = (valid & 1u) ? ld_shared_v4(raw + slot * kRawBytes + rope_src) : make_uint4(0, 0, 0, 0);
                rope[1] = (valid4 & 1u) ? ld_shared_v4(raw + slot * kRawBytes + rope_src + 4 * kLatentQ4RowBytes) : make_uint4(0, 0, 0, 0);
            }
            done_with(slot);
            next_slot();
            if (is_v) {
                ok = wait_warp(bar_raw_full + 8 * slot, raw_ph);
                if (!ok) break;
                read(code[2], code[3], scale[2], scale[3], my_chunk);
                done_with(slot);
                next_slot();
            }
            ok = wait_warp(bar_free + 8 * st, ((static_cast<uint32_t>(t) >> 1) & 1u) ^ 1u);
            if (!ok) break;
            uint32_t to = my_dst + st * buf_bytes;
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                const Q4Scale s0 = q4_scale_of(scale[0]), s1 = q4_scale_of(scale[1]);
                const uint32_t odd = (to + 4 * 128) ^ 64u;
                st_shared_v4(to, dequant8_q4(code[0].x, s0));
                st_shared_v4(to ^ 16u, dequant8_q4(code[0].y, s0));
                st_shared_v4(to ^ 32u, dequant8_q4(code[0].z, s0));
                st_shared_v4(to ^ 48u, dequant8_q4(code[0].w, s0));
                st_shared_v4(odd, dequant8_q4(code[1].x, s1));
                st_shared_v4(odd ^ 16u, dequant8_q4(code[1].y, s1));
                st_shared_v4(odd ^ 32u, dequant8_q4(code[1].z, s1));
                st_shared_v4(odd ^ 48u, dequant8_q4(code[1].w, s1));
                code[0] = code[2];
                code[1] = code[3];
                scale[0] = scale[2];
                scale[1] = scale[3];
                to += to_second;
            }
            if (!is_v) {
                st_shared_v4(rope_dst + st * kKBytes, rope[0]);
                st_shared_v4((rope_dst + st * kKBytes + 4 * 128) ^ 64u, rope[1]);
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(bar_full + 8 * st);
            if (!is_v) {                                      // K has no use for the other half: its turn is passed when it has landed
                ok = wait_warp(bar_raw_full + 8 * slot, raw_ph);
                if (!ok) break;
                done_with(slot);
                next_slot();
            }
        }
        if (!ok && lane == 0) give_up(DEV_TIMEOUT_GATHER);
    } else if (warp >= 4 && warp < 8) {
        // ------------------------------------------------------------ softmax and output
        // Warps q and q ^ 2 share 32 query rows: this one has the tile's rows 32 half .. 32 half + 31 of each and, of the output, value
        // columns 256 half .. 256 half + 255. They exchange the rows' maxima at every tile, so that both use the same reference.
        const int q = warp & 3, half = q >> 1;
        const int row = (q & 1) * 32 + lane;
        const uint32_t lane_base = tmem_base + (static_cast<uint32_t>(q * 32) << 16);
        uint8_t* const p_row = p_smem + row * 128;
        write_empty_units(p, group, q, lane, seq_rows, rows_of);
        // Both warps of a row leave the tile loop at the same barrier or not at all: `ok` is only acted upon there.
        while (walk.next(pc)) {
            const int n_rows = rows_of(pc.unit, seq, r0);
            if (ROWS == kCodes) {
                // Q's first blocks: this thread's row (both lane halves hold it) to tensor memory; the scores of the last piece are done. Rows
                // that are not ours become zeros: they only reach scores of rows that nobody reads.
                const uint4* src = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(p.a.q) + (seq * seq_rows + r0 + row) * (kLatentCols * 2));
                auto load_block = [&](int b, uint32_t (&r)[32]) {
#pragma unroll
                    for (int ch = 0; ch < 8; ++ch) {
                        const uint4 v = row < n_rows ? __ldg(src + b * 8 + ch) : make_uint4(0, 0, 0, 0);
                        r[4 * ch] = v.x; r[4 * ch + 1] = v.y; r[4 * ch + 2] = v.z; r[4 * ch + 3] = v.w;
                    }
                };
                uint32_t ra[32], rb[32];
                load_block(0, ra);
#pragma unroll 1
                for (int b = 0; b < kQT; b += 2) {
                    load_block(b + 1, rb);
                    __syncwarp();
                    tmem_st_32x32b_x32(lane_base + kColQ + b * 32, ra);
                    if (b + 2 < kQT) load_block(b + 2, ra);
                    __syncwarp();
                    tmem_st_32x32b_x32(lane_base + kColQ + (b + 1) * 32, rb);
                }
                tmem_st_wait();
                tcgen05_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(in_first(bar_q_ready));
            }
            const int64_t len = seq_len(seq);
            const int64_t base = first_row(p.a, seq);
            // positions [lo, sees) are seen by this row: those inside the cache, up to the row's own new token
            int sees = 0;
            if (row < n_rows) {
                int64_t n = len;
                if (!p.a.topk) n = min(len - (p.a.n_step - 1 - (r0 + row) / p.a.H), p.a.n_kv - base);
                sees = static_cast<int>(max(n, int64_t(0)));
            }
            const int lo = p.a.topk ? 0 : static_cast<int>(min(max(-base, int64_t(0)), int64_t(1) << 30));
            float m_ref = -INFINITY, l = 0.f;
            for (int i = 0; i < pc.n; ++i, ++tile) {
                const uint32_t st = tile & 1u, ph = (tile >> 1) & 1u;
                ok = ok && wait_warp(bar_s_full + 8 * st, ph);
                float x[32];
                float mt = -INFINITY;
                if (ok) {
                    tcgen05_fence_after_sync();
                    uint32_t s[32];
                    tmem_ld_32x32b_x32(lane_base + kColS + st * 32, s);
                    uint32_t usable = 0xFFFFFFFFu;
                    if (ROWS == kPicked)
                        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(usable) : "r"(smem_u32(const_cast<uint8_t*>(mask_smem)) + ((tile & 3u) * 2 + half) * 4) : "memory");
                    tmem_ld_wait(s);
                    tcgen05_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(in_first(bar_s_free + 8 * st));
#pragma unroll
                    for (int k = 0; k < 32; ++k) x[k] = __uint_as_float(s[k]);
                    if (p.sign != 1.f) {                                  // a negative or zero scale: what is scaled grows with the score
#pragma unroll
                        for (int k = 0; k < 32; ++k) x[k] *= p.sign;
                    }
                    const int at = (pc.t0 + i) * kTile + half * kHalf;
                    if (__any_sync(0xFFFFFFFFu, at + kHalf > sees || at < lo || usable != 0xFFFFFFFFu)) {
#pragma unroll
                        for (int k = 0; k < 32; ++k)
                            if (at + k >= sees || at + k < lo || !((usable >> k) & 1u)) x[k] = -INFINITY;
                    }
                    float m4[4];                                          // short chains
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        m4[k] = fmaxf(x[k], x[k + 4]);
#pragma unroll
                        for (int e = 8; e < 32; e += 8) m4[k] = fmaxf(m4[k], fmaxf(x[k + e], x[k + e + 4]));
                    }
                    mt = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * p.scale_log2;
                }
                swap[(st * 4 + q) * 32 + lane] = mt;
                ok = pair_of_warps_ok(1 + (q & 1), ok);
                if (!ok) break;
                mt = fmaxf(mt, swap[(st * 4 + (q ^ 2)) * 32 + lane]);
                float alpha = 1.f;
                bool move = false;
                if (mt > m_ref + kMoveThreshold) {                        // also the first usable score (m_ref = -inf)
                    alpha = m_ref == -INFINITY ? 0.f : exp2_fast(m_ref - mt);
                    m_ref = mt;
                    l *= alpha;
                    move = true;
                }
                const float ref = m_ref == -INFINITY ? 0.f : m_ref;
                float sum[4] = {0.f, 0.f, 0.f, 0.f};
                uint32_t pk[16];
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const float p0 = exp2_fast(__fmaf_rn(x[2 * k], p.scale_log2, -ref)), p1 = exp2_fast(__fmaf_rn(x[2 * k + 1], p.scale_log2, -ref));
                    sum[k & 3] += p0 + p1;
                    pk[k] = pack2(p0, p1);
                }
                l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
                // P's buffer is free when the product of the tile before the last has read it; a rescale of O waits for the last product
                ok = wait_warp(bar_pv_done + 8 * st, ph ^ 1u);
                if (i > 0 && __any_sync(0xFFFFFFFFu, move)) {
                    ok = ok && wait_warp(bar_pv_done + 8 * (st ^ 1u), ((tile - 1u) >> 1) & 1u);
                    if (ok) {
                        tcgen05_fence_after_sync();
#pragma unroll 1
                        for (int c = 0; c < 8; ++c) {
                            uint32_t o[32];
                            tmem_ld_32x32b_x32(lane_base + c * 32, o);
                            tmem_ld_wait(o);
#pragma unroll
                            for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * alpha);
                            tmem_st_32x32b_x32(lane_base + c * 32, o);
                        }
                        tmem_st_wait();
                    }
                }
                if (ok) {
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        *reinterpret_cast<uint4*>(p_row + st * kPBytes + (((half * 4 + v) ^ (row & 7)) << 4)) =
                            make_uint4(pk[4 * v], pk[4 * v + 1], pk[4 * v + 2], pk[4 * v + 3]);
                    fence_proxy_async_smem();
                    tcgen05_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(in_first(bar_p_ready + 8 * st));
                }
            }
            // the last product (tile - 1), and the other half's part of the sum
            ok = ok && wait_warp(bar_pv_done + 8 * ((tile - 1u) & 1u), ((tile - 1u) >> 1) & 1u);
            swap[(2 * 4 + q) * 32 + lane] = l;
            ok = pair_of_warps_ok(1 + (q & 1), ok);
            if (!ok) break;
            tcgen05_fence_after_sync();
            l += swap[(2 * 4 + (q ^ 2)) * 32 + lane];
            const float inv = l != 0.f ? 1.f / l : 0.f;                   // 0: the row saw nothing; a sum that is no number stays none
            const int64_t at_row = seq * seq_rows + r0 + row;
            const int64_t slot = ((static_cast<int64_t>(group) * 2 + (pc.t0 == 0 ? 1 : 0)) * 2 + rank) * kRows + row;
            // P's buffers are free now, and until both warps of a row have met at the next tile: a quarter for each warp to turn its rows in
            const uint32_t stage = smem_u32(p_smem) + q * 4096;
            const int first_row = (q & 1) * 32;
            if (pc.whole) {
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    uint4 v[8];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        uint32_t o[32];
                        tmem_ld_32x32b_x32(lane_base + c * 64 + e * 32, o);
                        tmem_ld_wait(o);
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            v[4 * e + k] = make_uint4(pack2(__uint_as_float(o[8 * k]) * inv, __uint_as_float(o[8 * k + 1]) * inv),
                                                      pack2(__uint_as_float(o[8 * k + 2]) * inv, __uint_as_float(o[8 * k + 3]) * inv),
                                                      pack2(__uint_as_float(o[8 * k + 4]) * inv, __uint_as_float(o[8 * k + 5]) * inv),
                                                      pack2(__uint_as_float(o[8 * k + 6]) * inv, __uint_as_float(o[8 * k + 7]) * inv));
                    }
                    store_rows(stage, lane, v, [&](int r, int i) -> uint4* {
                        return first_row + r < n_rows ? reinterpret_cast<uint4*>(p.out + (at_row - lane + r) * 512 + half * 256 + c * 64) + i : nullptr;
                    });
                }
            } else {
#pragma unroll 1
                for (int c = 0; c < 8; ++c) {
                    uint32_t o[32];
                    tmem_ld_32x32b_x32(lane_base + c * 32, o);
                    tmem_ld_wait(o);
                    uint4 v[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        v[k] = make_uint4(__float_as_uint(__uint_as_float(o[4 * k]) * inv), __float_as_uint(__uint_as_float(o[4 * k + 1]) * inv),
                                          __float_as_uint(__uint_as_float(o[4 * k + 2]) * inv), __float_as_uint(__uint_as_float(o[4 * k + 3]) * inv));
                    store_rows(stage, lane, v, [&](int r, int i) -> uint4* {
                        return first_row + r < n_rows ? reinterpret_cast<uint4*>(p.part_out + (slot - lane + r) * 512 + half * 256 + c * 32) + i : nullptr;
                    });
                }
            }
            tcgen05_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(in_first(bar_o_free));
            if (half == 0 && row < n_rows) {
                const float lse = l != 0.f ? (m_ref + log2f(l)) * 0.6931471805599453f : -INFINITY;
                if (!pc.whole) p.part_lse[slot] = lse;
                else if (p.lse) p.lse[at_row] = lse;
            }
        }
        if (!ok && lane == 0) give_up(DEV_TIMEOUT_EPILOGUE);
    }

    // ---------------------------------------------------------------- teardown: neither CTA leaves while the other may still reach it
    __syncwarp();
    if (*abort_flag) {                       // copies may still be in flight: let them land before the CTA's memory goes
        const long long t0 = clock64();
        while (clock64() - t0 < 2000000LL) __nanosleep(1000);
    }
    tcgen05_fence_before_sync();
    __syncthreads();
    cluster_sync();
    if (warp == 0) {
        tcgen05_fence_after_sync();
        tmem_dealloc_pair(tmem_base, 512);
    }
}

}  // namespace

cudaError_t launch_latent_attn_pair(const LatentMaps& maps, const Params& p, cudaStream_t stream) {
    auto go = [&](auto kernel, Rows rows, int warps) -> cudaError_t {
        if (cudaError_t e = ensure_max_dynamic_smem(reinterpret_cast<const void*>(kernel), smem_bytes(rows)); e != cudaSuccess) return e;
        if (rows == kPicked) return launch_behind(kernel, p.groups * 2, warps * 32, smem_bytes(rows), stream, maps.q, maps.k, maps.rope, maps.v, p);
        kernel<<<static_cast<unsigned>(p.groups * 2), warps * 32, smem_bytes(rows), stream>>>(maps.q, maps.k, maps.rope, maps.v, p);
        return cudaGetLastError();
    };
    if (!p.a.q4) return go(latent_attn_pair_kernel<kBf16>, kBf16, kWarpsBf16);
    return p.a.topk ? go(latent_attn_pair_kernel<kPicked>, kPicked, kWarpsQ4) : go(latent_attn_pair_kernel<kCodes>, kCodes, kWarpsQ4);
}

}  // namespace idxc
