// Attention of new tokens over their requests' pages of keys and values, H / H_kv query heads to a key head:
//     x[s] = scale <q, k_s> over the visible keys s,   out = sum_s softmax(x)[s] v_s,   lse = log sum_s exp(x[s])
// over all pages of a request, or over the pages that a selection names for each (request, key head).
//
// A unit is a (request, key head). Few units of few tiles: a cluster of up to 8 CTAs takes a unit and joins its parts over distributed shared
// memory, one launch in all.
//
// Measured (graph replays, one B200): 32 requests of 4K to 32K bf16 keys, 64 heads over 8: 352 us, 6.9 TB/s of what has to be read; 8 requests of 131072
// 8-bit keys: 352 to 371 us from run to run, 6.3 to 6.0 TB/s; 8 x 32768 with 16 / 32 rows a key head: bf16 6.4 / 6.2, 8 bits 5.4 / 3.4 TB/s; one request of 777
// keys: 6.5 us.
//
// What bounds it: a key and a value of d columns are 4 d bytes (bf16) and 4 d flops a query row; with the 1 to 32 rows that share a key head
// in a decode step that is 1 to 32 flops a byte, far below the tensor cores' 200: HBM. So the design serves the copies: a ring of 64- or 128-key tiles
// of K and V (32 KB in bf16 with d = 128), filled by TMA with whole pages or 16-key pieces of them, and as few instructions a tile as will do.
//
// Keys are the M = 16 of the matrix instructions, query rows their N = 8: S^T = K Q^T and O^T = V^T P^T. Up to 8 rows (a group of 8 heads) then waste
// nothing, K and V are read from shared memory once for any number of rows, and scores, softmax and output stay in registers. (With rows as M, 8 rows were half
// padding, and 64 keys in 8 bits took 1740 instructions instead of 1390. tcgen05's M = 64 or 128 with rows as N would fit too, but its scores would cross
// tensor memory twice a tile, a latency that several resident CTAs would have to hide.) P^T comes out of the scores' registers by an 8 x 8 transposition.
//
// Up to 32 rows (more: paged_attn_rows.cu): 4 warps, each 16 or 32 keys of a tile with its own running reference and sum; 2 or 3 CTAs an SM hide each
// other's segment ends. The warps' parts meet once at a segment's end, in shared memory. The tiles of all
// units, end to end, are cut into runs of equal cost, a run a CTA, which finds it from the lengths on the device;
// segments cut by a run's end go to the workspace in fp32 and through a merge kernel. All sums have an order fixed by the sizes, so results
// repeat bit for bit.
//
// e4m3 rows: codes become f16 (exact) on the way to the registers, with q as f16 times a power of two a row (its largest element in [1, 2); what
// falls below f16's range is below 2^-25 of that, an fp32 rounding). The value's scale goes into the probability, whose reference is the running
// maximum of x + log2(scale), rounded up: probability times scale then stays in f16's range however the scales differ.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "kernels.h"
#include "paged_attn.cuh"
#include "ptx_sm100.cuh"

namespace idxc {
using namespace paged;
namespace {

constexpr int kProducerRegs = 40;
// Rows of a key head up to which this kernel is the faster one. (8 x 32768 keys, 8 key heads, d = 128 / 64. bf16: 32 rows 173 / 99 us here, 64 rows, with 8 warps
// of which two shared keys, 240 / 183, and 183 / 111 by paged_attn_rows.cu. 8 bits: 32 rows 159 / 111 here and 215 / 161 there, 64 rows 305 / 227 and 232 / 182.)
constexpr int kRowsHere = 32;
// Tiles of a CTA up to which few units are given to clusters. (bf16, 8 key heads, d = 128, one request of 777 / 2000 / 4000 / 8000 keys: 9.3 / 11.1 / 12.7 /
// 13.9 us by runs and a merge, 6.1 / 7.5 / 10.4 / 16.4 by clusters, with 2, 4, 8 and 16 tiles a CTA.)
constexpr int kJoinTiles = 8;
// Tiles above an equal share that a cut and the merge cost. (64 pages of 32 for 16 requests and 8 key heads, 8 rows: bf16, 16 tiles a CTA where 14 are a share, 30
// us by runs, 26.6 by clusters of two; 8 bits, 16 where 9 are, 20.4 and 23.0. 32 pages of 64 in 8 bits for 100 requests and 4 heads, 32 and 29: 53 and 40.)
constexpr int kJoinSlack = 5;
// Log2 units by which a score may pass its row's reference before that moves. In bf16 up to 16 rows the reference is the maximum: the largest
// probability is then 1, which bf16 holds exactly (error of out against 64 bits for 16 requests over 64 pages: 2.2e-3 with 8, 1.8e-3 with 0, of which
// 1.7e-3 are the output's own rounding). With 32 rows a warp some reference moves at most steps, and that costs an eighth of the time (96 requests
// of 16 heads and 4 tokens: 33.5 us with 8, 37.4 with 0). f16 of 8-bit rows is exact enough either way.
template <bool FP8, int NR>
constexpr float kSlack = FP8 || NR == 4 ? 8.f : 0.f;
__device__ __forceinline__ uint32_t ld_shared_u32(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
// An 8 x 8 matrix of 16-bit elements, lane 4 g + j holding elements 2 j, + 1 of row g, transposed.
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ void st_shared_v2(uint32_t addr, uint32_t x, uint32_t y) {
    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(addr), "r"(x), "r"(y) : "memory");
}
// The two barriers of a cluster that joins its parts, for the warps that have no share in that: parts are there; parts have been read.
__device__ __forceinline__ void leave_cluster() {
    cluster_sync();
    cluster_sync();
}
__device__ __forceinline__ float2 ld_cluster_f32x2(uint32_t addr) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
    return v;
}
template <int WARPS>
__device__ __forceinline__ void consumers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(WARPS * 32) : "memory"); }

// ---------------------------------------------------------------- work
struct Walk {
    const Params& p;
    int b, x, left, nt;
    __device__ __forceinline__ Walk(const Params& q, const Run& r) : p(q), b(r.b), x(r.x), left(r.n), nt(r.n > 0 && !q.join ? tiles_of(q, r.b) : 0) {}
    __device__ __forceinline__ bool next(Segment& s) {
        if (p.join) {                            // this CTA's share of its cluster's unit, which may be none; once
            if (left == 0) return false;
            left = 0;
            const int unit = blockIdx.x / p.join, rank = blockIdx.x % p.join;
            s.b = unit / p.a.c.H_kv;
            s.head = unit - s.b * p.a.c.H_kv;
            s.nt = tiles_of(p, s.b);
            s.t0 = static_cast<int>(static_cast<unsigned>(s.nt) * rank / p.join);
            s.n = static_cast<int>(static_cast<unsigned>(s.nt) * (rank + 1) / p.join) - s.t0;
            return true;
        }
        const int units = p.units;
        while (left > 0) {
            while (x == length_of_unit(nt) * units) {       // the request's end (or one without tiles); more follow
                nt = tiles_of(p, ++b);
                x = 0;
            }
            const int len = nt + kSegmentTiles;
            s.b = b;
            const int unit = x / len, from = x - unit * len, n = min(len - from, left);
            s.head = unit * p.heads + static_cast<int>(blockIdx.x) % p.heads;
            x += n;
            left -= n;
            s.t0 = max(from - kSegmentTiles, 0);
            s.n = max(from + n - kSegmentTiles, 0) - s.t0;
            s.nt = nt;
            if (s.n > 0) return true;
        }
        return false;
    }
};

// ---------------------------------------------------------------- shared memory
// NR blocks of 8 query rows.
// With 32 rows a warp the output alone is 128 registers of d = 128: registers are then handed out unevenly, by warpgroups (three idle warps fill
// up the producer's): the launch's 128 a thread, of which the producer's warpgroup keeps 40.
template <int D, bool FP8, int NR>
struct Layout {
    static constexpr int kWarps = 4;                                   // consumers; they share every tile
    static constexpr bool kUneven = NR * D == 512;
    static constexpr int kThreads = (kWarps + (kUneven ? 4 : 1)) * 32;
    static constexpr int kCtas = NR == 1 && FP8 ? 3 : 2;               // of an SM
    static constexpr int kConsumerRegs = 216;
    static_assert(128 * kProducerRegs + kWarps * 32 * kConsumerRegs <= (kWarps + 4) * 32 * 128, "shares of the launch's registers");
    // Keys of a tile: 18 to 36 KB, so that a tile's fixed costs (barriers, votes, the producer's turn) stay small beside its bytes, as far as a ring
    // of three leaves room. (One request length of 32768 and 8 key heads, 8 rows: d = 64 in bf16 108 us with 64 keys and three CTAs, 91 with these.)
    static constexpr int kTile = (D == 64 && (FP8 || NR < 4)) || (FP8 && NR == 2) ? 128 : 64;
    static constexpr int kRows = 8 * NR;                               // query rows of a CTA
    static constexpr int kKeys = kTile / kWarps;                       // keys of a tile that a warp takes
    static constexpr int kTileBytes = kTile * D * (FP8 ? 1 : 2);
    static constexpr int kStageBytes = (2 * kTileBytes + (FP8 ? 8 * kTile : 0) + 1023) / 1024 * 1024;      // K, V, scales of K and of V: swizzled rows
                                                                                                           // begin on multiples of 1024 bytes
    static constexpr int kSlice = NR == 1 ? 64 : (NR == 2 ? 32 : 16);  // columns of the output that go through shared memory at a time
    static constexpr int kPitch = kSlice + 4;                          // floats between rows there: no bank conflicts
    static constexpr int kQBytes = kRows * D * 2;
    static constexpr int kRedBytes = kWarps * kRows * kPitch * 4;
    static constexpr int kShared = kQBytes > kRedBytes ? kQBytes : kRedBytes;  // q, and the output's slices when q is done with
    static constexpr int kMlBytes = kWarps * kRows * 8;
    static constexpr int kSmall = 1024 + 1536;                         // alignment of the stages; barriers, positions, a number per row
    static constexpr int kLimit = (233472 - kCtas * (1024 + 128)) / kCtas;     // an SM's, without what the system and static arrays take
    static constexpr int kFit = (kLimit - kSmall - kShared - kMlBytes) / kStageBytes;
    // Every warp sees every phase of every stage's barrier. (If warps took tiles in turn, one could come to a stage's barrier while the tile
    // before its own is still on the way, and take the parity of the one before that for its own.)
    static constexpr int kStages = kFit > 24 ? 24 : kFit;
    static constexpr int kBytes = kSmall + kStages * kStageBytes + kShared + kMlBytes;
    static_assert(kStageBytes % 1024 == 0 && kTileBytes % 1024 == 0, "the swizzle goes by the address");
    static_assert(kKeys % 16 == 0 && kStages >= 3, "whole steps of 16 keys, a ring of at least three tiles");
    static_assert(kRows * (D * 4 + 8) <= kStages * kStageBytes, "a CTA's part of a cluster's unit");
    static_assert(kStages * (16 + 32) + kRows * 4 + 16 <= 1536 && kTile <= 128, "small words");
};

// Byte offset of 16-byte chunk `c` of row `r` in a tile whose rows are at most 128 bytes (wider ones lie in blocks of 128).
template <int ROW_BYTES, int TILE>
__device__ __forceinline__ uint32_t chunk_at(int r, int c) {
    if (ROW_BYTES >= 128) return (c >> 3) * (TILE * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4);
    return r * 64 + ((c ^ ((r >> 1) & 3)) << 4);
}

template <int D, bool FP8, int NR>
__global__ void __launch_bounds__((Layout<D, FP8, NR>::kThreads), (Layout<D, FP8, NR>::kCtas))
paged_attn_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const __grid_constant__ Params p) {
    using L = Layout<D, FP8, NR>;
    constexpr int ROWB = D * (FP8 ? 1 : 2);      // bytes of a cached row
    constexpr int NS = L::kStages, W = L::kWarps;
    extern __shared__ uint8_t raw[];
    const uint32_t base = smem_u32(raw);
    const uint32_t stages = (base + 1023u) & ~1023u;
    const uint32_t q_s = stages + NS * L::kStageBytes;
    const uint32_t red_s = q_s;
    const uint32_t join_s = stages;              // [rows][D] output and [rows] (maximum, sum) of a CTA whose cluster joins them, when its tiles are done with
    const uint32_t ml_s = q_s + L::kShared;      // [parts][rows] (maximum, sum) of a warp, then (factor, -)
    const uint32_t bars = ml_s + L::kMlBytes;    // full[NS], empty[NS]
    const uint32_t pos_s = bars + NS * 16;       // [NS][8] position of the first key of each piece, -1: none
    const uint32_t row_s = pos_s + NS * 32;      // [rows] power of two taken out of a row of q; at the end what the row is multiplied by
    const uint32_t flag_s = row_s + L::kRows * 4;
    __shared__ int scratch[18];
    volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(raw + (flag_s - base));

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < NS; ++s) {
            mbar_init(bars + 8 * s, 1);
            mbar_init(bars + 8 * (NS + s), W);
        }
        *abort_flag = 0;
        fence_mbar_init();
        if (p.a.c.n_pages > 0) {                 // (a cache without pages has no maps)
            tma_prefetch_desc(&k_map);
            tma_prefetch_desc(&v_map);
        }
    }
    let_next_start();
    wait_for_previous();
    Run run{0, 0, 1, 0};
    if (p.join) __syncthreads();
    else run = find_run(p, scratch, [&](int b) { return length_of_unit(tiles_of(p, b)) * p.units; });      // (its barriers publish the mbarriers too)
    const PagedAttnArgs& a = p.a;

    if (warp >= W) {
        if (L::kUneven) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kProducerRegs));
        if (warp > W) {
            if (p.join > 1) leave_cluster();
            return;
        }
        // ------------------------------------------------------------ producer: pieces of pages into the ring
        constexpr int kTileLog2 = L::kTile == 64 ? 6 : 7;
        const int piece = 1 << p.piece_log2, per_tile_log2 = kTileLog2 - p.piece_log2, per_tile = 1 << per_tile_log2;
        const uint32_t piece_bytes = static_cast<uint32_t>(piece) * (2 * ROWB + (FP8 ? 8 : 0));
        const int P = a.c.page_size;
        int it = 0;
        Walk walk(p, run);
        Segment s;
        while (walk.next(s)) {
            const int len = length_of(a, s.b);
            const int head = s.head;
            const int32_t* table = a.table + static_cast<int64_t>(s.b) * a.ld_table;
            const int32_t* sel = a.pages ? a.pages + (static_cast<int64_t>(s.b) * a.c.H_kv + head) * a.n_sel : nullptr;
            const int n_entries = (len + P - 1) / P;      // pages of the request; with a selection min(n_sel, that) entries are looked at
            const int most = sel ? min(a.n_sel, n_entries) : n_entries;
            const int n_pieces = s.n << per_tile_log2;
            struct Where { int page, off, pos; };
            auto locate = [&](int i) -> Where {           // piece i of the segment
                Where w{0, 0, -1};
                if (i < n_pieces) {
                    const unsigned v = static_cast<unsigned>(s.t0) * L::kTile + (static_cast<unsigned>(i) << p.piece_log2);
                    const unsigned e = v / static_cast<unsigned>(P);
                    w.off = static_cast<int>(v - e * P);
                    if (static_cast<int>(e) < most) {
                        const int logical = sel ? sel[e] : static_cast<int>(e);
                        if (logical >= 0 && logical < n_entries) {
                            const int pos = logical * P + w.off;
                            w.page = table[logical];
                            if (pos < len && w.page >= 0 && w.page < a.c.n_pages) w.pos = pos;
                        }
                    }
                }
                return w;
            };
            Where next = locate(lane);
            for (int i0 = 0; i0 < n_pieces; i0 += 32) {
                const Where now = next;
                if (i0 + 32 < n_pieces) next = locate(i0 + 32 + lane);
                const int n_here = min(32, n_pieces - i0) >> per_tile_log2;      // tiles
                for (int t = 0; t < n_here; ++t, ++it) {
                    const int st = it % NS;
                    if (it >= NS && !mbar_wait(bars + 8 * (NS + st), ((it / NS) & 1) ^ 1, abort_flag)) {
                        if (lane == 0) {
                            *abort_flag = 1;
                            atomicCAS(p.status, DEV_OK, DEV_TIMEOUT_PRODUCER);
                        }
                        goto drain;
                    }
                    const bool mine = (lane >> per_tile_log2) == t;
                    const int in_tile = lane & (per_tile - 1);
                    const uint32_t who = __ballot_sync(0xFFFFFFFFu, mine && now.pos >= 0);
                    if (mine) asm volatile("st.shared.b32 [%0], %1;" ::"r"(pos_s + st * 32 + in_tile * 4), "r"(now.pos) : "memory");
                    __syncwarp();
                    const uint32_t full = bars + 8 * st;
                    if (lane == 0) mbar_arrive_expect_tx(full, __popc(who) * piece_bytes);
                    __syncwarp();
                    if (mine && now.pos >= 0) {
                        const uint32_t k_to = stages + st * L::kStageBytes, v_to = k_to + L::kTileBytes;
                        constexpr int INNER = ROWB >= 128 ? 128 : ROWB;          // bytes of a row of one copy
                        const uint32_t at = in_tile * piece * INNER;
#pragma unroll
                        for (int h = 0; h < ROWB / INNER; ++h) {
                            tma_load_4d(k_to + h * (L::kTile * INNER) + at, &k_map, full, h * 64, now.off, head, now.page);
                            tma_load_4d(v_to + h * (L::kTile * INNER) + at, &v_map, full, h * 64, now.off, head, now.page);
                        }
                        if (FP8) {
                            const int64_t from = (static_cast<int64_t>(now.page) * a.c.H_kv + head) * P + now.off;
                            const uint32_t sc = v_to + L::kTileBytes + in_tile * piece * 4;
                            bulk_load_1d(sc, a.c.k_scale + from, piece * 4, full);
                            bulk_load_1d(sc + 4 * L::kTile, a.c.v_scale + from, piece * 4, full);
                        }
                    }
                }
            }
        }
    drain:
        // The copies of the last tiles have landed when their consumers have seen them; a producer that gave up waits for its own.
        if (*abort_flag) {
            const int from = it > NS ? it - NS : 0;
            for (int i = from; i < it; ++i) {
                const long long t0 = clock64();
                while (!mbar_try_wait(bars + 8 * (i % NS), (i / NS) & 1) && clock64() - t0 < kWaitCycleBudget) {}
            }
        }
        __syncwarp();
        if (p.join > 1) leave_cluster();
        return;
    }

    // ---------------------------------------------------------------- consumers
    if (L::kUneven) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(L::kConsumerRegs));
    const int g = lane >> 2, j = lane & 3;       // of a fragment: key (or output column) g and g + 8, query rows 2 j and 2 j + 1
    const int rows_all = a.n_step * a.group;
    constexpr int NT = D / 16;                   // output fragments of 16 columns
    constexpr int KB = NR <= 2 && L::kKeys >= 32 ? 2 : 1;      // blocks of 16 keys in a step
    constexpr int CH = NR * KB == 1 ? 2 : 1;     // sums that a block's scores are formed in
    constexpr bool kQRegs = NR * D <= 128;              // q's fragments stay in registers, and the next segment's q is on its way early
    constexpr int QV = L::kRows * (D / 8) / (W * 32) > 0 ? L::kRows * (D / 8) / (W * 32) : 1;      // vectors of q a thread brings
    constexpr int Q_THREADS = L::kRows * (D / 8) < W * 32 ? L::kRows * (D / 8) : W * 32;

    auto load_q = [&](const Segment& s, uint4(&q)[QV]) {              // zeros behind the last row
        const int head = s.head;
#pragma unroll
        for (int u = 0; u < QV; ++u) {
            const int i = threadIdx.x + u * W * 32, r = i / (D / 8), c = i - r * (D / 8);
            q[u] = make_uint4(0u, 0u, 0u, 0u);
            if (threadIdx.x < Q_THREADS && r < rows_all) {
                const int step = r / a.group, h = r - step * a.group;
                q[u] = reinterpret_cast<const uint4*>(a.q + (static_cast<int64_t>(s.b) * a.n_step + step) * a.q_stride +
                                                      static_cast<int64_t>(head * a.group + h) * D)[c];
            }
        }
    };
    int it = 0;
    bool ok = true;
    Walk walk(p, run);
    Segment s, after;
    int4 owner = make_int4(-1, 0, 0, 0);
    uint4 q_next[QV];
    bool more = walk.next(after);
    if (kQRegs && more) load_q(after, q_next);
    while (more) {
        s = after;
        if (!kQRegs) load_q(s, q_next);
        const int len = length_of(a, s.b);
        const int head = s.head, n_rows = rows_all;
        const bool whole = s.t0 == 0 && s.n == s.nt && p.join <= 1;
        if (threadIdx.x < Q_THREADS) {
#pragma unroll
            for (int u = 0; u < QV; ++u) {
                const int i = threadIdx.x + u * W * 32, r = i / (D / 8), c = i - r * (D / 8);
                const uint32_t row_at = q_s + r * (D * 2);
                const uint4 x = q_next[u];
                if (!FP8) {
                    st_shared_v4(row_at + ((c ^ (r & 7)) << 4), x);
                } else {
                    // the D / 8 threads of a row are neighbours in a warp
                    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
                    float f[8], top = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        f[e] = __uint_as_float(e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
                        top = fmaxf(top, fabsf(f[e]));
                    }
#pragma unroll
                    for (int o = D / 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
                    const int exponent = min(max(static_cast<int>(__float_as_uint(top) >> 23), 1), 253);      // top in [2^(exponent - 127), 2 of that)
                    const float down = __uint_as_float(static_cast<uint32_t>(254 - exponent) << 23);
                    if (c == 0) st_shared_f32(row_s + r * 4, __uint_as_float(static_cast<uint32_t>(exponent) << 23));
                    uint32_t h[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) h[e] = pack_f16(f[2 * e] * down, f[2 * e + 1] * down);
                    // Of 16 columns lane j of a fragment takes 4 j .. 4 j + 3 (the four codes of a register of K): pairs 0 and 1 of each four
                    // go to places 2 j and 2 j + 8.
                    const int block = c >> 1, odd = c & 1;             // 16 columns; the second eight of them
                    st_shared_v2(row_at + (((2 * block) ^ (r & 7)) << 4) + odd * 8, h[0], h[2]);
                    st_shared_v2(row_at + (((2 * block + 1) ^ (r & 7)) << 4) + odd * 8, h[1], h[3]);
                }
            }
        }
        consumers_sync<W>();

        // B fragments of q for two steps of 16 columns and a block of 8 rows: matrices of 8 rows x 8 columns side by side.
        auto q_frag = [&](int nr, int c4, uint32_t(&f)[4]) {
            const int r = nr * 8 + (lane & 7), c = c4 * 4 + (lane >> 3);
            ldmatrix_x4(q_s + r * (D * 2) + ((c ^ (r & 7)) << 4), f);
        };
        uint32_t qf[kQRegs ? NR : 1][kQRegs ? D / 32 : 1][4];
        if (kQRegs) {
#pragma unroll
            for (int nr = 0; nr < NR; ++nr)
#pragma unroll
                for (int c4 = 0; c4 < D / 32; ++c4) q_frag(nr, c4, qf[kQRegs ? nr : 0][kQRegs ? c4 : 0]);
        }
        int sees[NR][2];                         // keys that rows 2 j, 2 j + 1 see
        float row_scale[NR][2], m[NR][2], l[NR][2];
        float o[NR][NT][4];
#pragma unroll
        for (int nr = 0; nr < NR; ++nr)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = nr * 8 + 2 * j + e;
                sees[nr][e] = len - (a.n_step - 1 - min(r / a.group, a.n_step - 1));
                row_scale[nr][e] = FP8 ? p.scale_log2 * ld_shared_f32(row_s + r * 4) : p.scale_log2;
                m[nr][e] = -INFINITY;
                l[nr][e] = 0.f;
            }
        const int sees_least = len - (a.n_step - 1);      // (of the request's first token)
#pragma unroll
        for (int nr = 0; nr < NR; ++nr)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[nr][n][e] = 0.f;

        for (int t = 0; t < s.n; ++t) {
            const int st = (it + t) % NS;
            if (ok && !mbar_wait(bars + 8 * st, ((it + t) / NS) & 1, abort_flag)) {
                if (lane == 0) {
                    *abort_flag = 1;
                    atomicCAS(p.status, DEV_OK, DEV_TIMEOUT_MMA);
                }
                ok = false;
            }
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (!ok) break;
            const uint32_t k_at = stages + st * L::kStageBytes, v_at = k_at + L::kTileBytes, sc_at = v_at + L::kTileBytes;
#pragma unroll
            for (int step = 0; step < L::kKeys / (16 * KB); ++step) {
                int key0[KB], at[KB];                      // first key of each 16, and its position
                int first = INT32_MAX, last = 0;
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) {
                    key0[kb] = warp * L::kKeys + (step * KB + kb) * 16;
                    const int pc = key0[kb] >> p.piece_log2;
                    at[kb] = static_cast<int>(ld_shared_u32(pos_s + st * 32 + pc * 4));
                    at[kb] = at[kb] < 0 ? INT32_MAX / 2 : at[kb] + (key0[kb] - (pc << p.piece_log2));
                    first = min(first, at[kb]);
                    last = max(last, at[kb] + 16);
                }
                if (L::kTile > 64 && first >= len) continue;           // none of them is there
                const bool clean = last <= sees_least;
                if (!clean) {
                    // Rows of V that no token sees meet probability 0 and may hold anything: they are cleared.
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb)
                        if (at[kb] + (lane & 15) >= len) {
                            const int r = key0[kb] + (lane & 15);
#pragma unroll
                            for (int c = 0; c < ROWB / 16; c += 2) st_shared_v4(v_at + chunk_at<ROWB, L::kTile>(r, c + (lane >> 4)), make_uint4(0u, 0u, 0u, 0u));
                            if (FP8) st_shared_f32(sc_at + 4 * L::kTile + r * 4, 1.f);
                            fence_proxy_async_smem();      // (the next copy into these rows comes from the asynchronous proxy)
                        }
                    __syncwarp();
                }
                // scores: A fragments straight from K's rows, (keys 0-7, 8-15) x two 16-byte chunks an ldmatrix; with few independent sums each is
                // formed in two, which halves the chain of dependent instructions
                float x[KB][NR][CH][4];
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int nr = 0; nr < NR; ++nr)
#pragma unroll
                        for (int e = 0; e < 4 * CH; ++e) x[kb][nr][e >> 2][e & 3] = 0.f;
#pragma unroll
                for (int c4 = 0; c4 < D / 32; ++c4)                    // 32 columns: two steps of 16
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb) {
                        uint32_t ka[2][4];
                        if (!FP8) {
#pragma unroll
                            for (int u = 0; u < 2; ++u)
                                ldmatrix_x4(k_at + chunk_at<ROWB, L::kTile>(key0[kb] + (lane & 15), c4 * 4 + 2 * u + (lane >> 4)), ka[u]);
                        } else {
                            uint32_t raw4[4];
                            ldmatrix_x4(k_at + chunk_at<ROWB, L::kTile>(key0[kb] + (lane & 15), c4 * 2 + (lane >> 4)), raw4);
#pragma unroll
                            for (int u = 0; u < 2; ++u)
#pragma unroll
                                for (int h = 0; h < 2; ++h) {          // keys g and g + 8: four codes each
                                    ka[u][h] = e4m3x2_to_f16x2(raw4[2 * u + h] & 0xFFFFu);
                                    ka[u][2 + h] = e4m3x2_to_f16x2(raw4[2 * u + h] >> 16);
                                }
                        }
#pragma unroll
                        for (int nr = 0; nr < NR; ++nr) {
                            uint32_t qb[4];
                            if (kQRegs) {
#pragma unroll
                                for (int e = 0; e < 4; ++e) qb[e] = qf[kQRegs ? nr : 0][kQRegs ? c4 : 0][e];
                            } else {
                                q_frag(nr, c4, qb);
                            }
                            mma_16816<FP8>(x[kb][nr][0], ka[0], qb[0], qb[1]);
                            mma_16816<FP8>(x[kb][nr][CH - 1], ka[1], qb[2], qb[3]);
                        }
                    }
                // softmax: element 2 h + e is key g + 8 h, row 2 j + e
                float v_sc[KB][2], y[KB][NR][4], top[NR][2];
                bool moved = false;
#pragma unroll
                for (int nr = 0; nr < NR; ++nr) top[nr][0] = top[nr][1] = -INFINITY;
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) {
                    float k_sc[2] = {1.f, 1.f}, above[2] = {0.f, 0.f};
                    if (FP8) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            k_sc[h] = ld_shared_f32(sc_at + (key0[kb] + g + 8 * h) * 4);
                            v_sc[kb][h] = ld_shared_f32(sc_at + 4 * L::kTile + (key0[kb] + g + 8 * h) * 4);
                            above[h] = log2_above(v_sc[kb][h]);
                            v_sc[kb][h] *= kF16Head;
                        }
                    }
#pragma unroll
                    for (int nr = 0; nr < NR; ++nr)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            float v = (CH == 2 ? x[kb][nr][0][e] + x[kb][nr][CH - 1][e] : x[kb][nr][0][e]) * row_scale[nr][e & 1];
                            if (FP8) v *= k_sc[e >> 1];
                            if (!clean && at[kb] + g + 8 * (e >> 1) >= sees[nr][e & 1]) v = -INFINITY;
                            y[kb][nr][e] = v;
                            top[nr][e & 1] = fmaxf(top[nr][e & 1], FP8 ? v + above[e >> 1] : v);
                        }
                }
#pragma unroll
                for (int nr = 0; nr < NR; ++nr) moved |= !(top[nr][0] <= m[nr][0] + kSlack<FP8, NR>) | !(top[nr][1] <= m[nr][1] + kSlack<FP8, NR>);
                if (__any_sync(0xFFFFFFFFu, moved)) {      // (rare behind a segment's first keys)
#pragma unroll
                    for (int nr = 0; nr < NR; ++nr)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float v = fmaxf(m[nr][e], top[nr][e]);
#pragma unroll
                            for (int d = 4; d < 32; d <<= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, d));
                            const float f = exp2_fast(m[nr][e] - (v == -INFINITY ? 0.f : v));
                            m[nr][e] = v;
                            l[nr][e] *= f;
#pragma unroll
                            for (int n = 0; n < NT; ++n) {
                                o[nr][n][e] *= f;
                                o[nr][n][2 + e] *= f;
                            }
                        }
                }
                uint32_t pb[KB][NR][2];
#pragma unroll
                for (int nr = 0; nr < NR; ++nr) {
                    const float use[2] = {m[nr][0] == -INFINITY ? 0.f : m[nr][0], m[nr][1] == -INFINITY ? 0.f : m[nr][1]};
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb) {
                        float* v = y[kb][nr];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            v[e] = exp2_fast(v[e] - use[e & 1]);
                            l[nr][e & 1] += v[e];
                            if (FP8) v[e] *= v_sc[kb][e >> 1];
                        }
                        pb[kb][nr][0] = transpose_8x8(FP8 ? pack_f16(v[0], v[1]) : pack_bf16(v[0], v[1]));
                        pb[kb][nr][1] = transpose_8x8(FP8 ? pack_f16(v[2], v[3]) : pack_bf16(v[2], v[3]));
                    }
                }
                // output: A fragments are V's rows transposed
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int c2 = 0; c2 < ROWB / 32; ++c2) {
                        uint32_t va[4];
                        if (!FP8) {
                            // (keys 0-7; columns 0-7, 8-15), then keys 8-15
                            ldmatrix_x4_trans(v_at + chunk_at<ROWB, L::kTile>(key0[kb] + (lane & 7) + (lane >> 4) * 8, 2 * c2 + (lane >> 3 & 1)), va);
#pragma unroll
                            for (int nr = 0; nr < NR; ++nr) mma_16816<false>(o[nr][c2 % NT], va, pb[kb][nr][0], pb[kb][nr][1]);
                        } else {
                            uint32_t vb[4];                // (keys 0-7, 8-15) of a 16-byte chunk, then of the next
                            ldmatrix_x4_trans(v_at + chunk_at<ROWB, L::kTile>(key0[kb] + (lane & 15), 2 * c2 + (lane >> 4)), vb);
#pragma unroll
                            for (int u = 0; u < 2; ++u) {
                                // A register holds columns 2 g, 2 g + 1 of keys 2 j, 2 j + 1: the even column's two keys become row g of the fragment,
                                // the odd one's row g + 8.
                                const uint32_t w0 = __byte_perm(vb[2 * u], 0, 0x3120), w1 = __byte_perm(vb[2 * u + 1], 0, 0x3120);
                                va[0] = e4m3x2_to_f16x2(w0 & 0xFFFFu);
                                va[1] = e4m3x2_to_f16x2(w0 >> 16);
                                va[2] = e4m3x2_to_f16x2(w1 & 0xFFFFu);
                                va[3] = e4m3x2_to_f16x2(w1 >> 16);
#pragma unroll
                                for (int nr = 0; nr < NR; ++nr) mma_16816<true>(o[nr][(2 * c2 + u) % NT], va, pb[kb][nr][0], pb[kb][nr][1]);
                            }
                        }
                    }
            }
            fence_proxy_async_smem();                      // (this warp's loads before the copies that refill the stage)
            __syncwarp();
            if (lane == 0) mbar_arrive(bars + 8 * (NS + st));
        }
        it += s.n;
        more = walk.next(after);
        if (kQRegs && more) load_q(after, q_next);         // (on the way while the warps' parts are joined)

        // ------------------------------------------------------------ the warps' parts of the segment joined
#pragma unroll
        for (int nr = 0; nr < NR; ++nr)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l[nr][e] += __shfl_xor_sync(0xFFFFFFFFu, l[nr][e], d);
                if (g == 0) st_shared_f32x2(ml_s + (warp * L::kRows + nr * 8 + 2 * j + e) * 8, m[nr][e], l[nr][e]);
            }
        consumers_sync<W>();
        const int64_t piece_row = (static_cast<int64_t>(blockIdx.x) * 2 + (s.t0 == 0 ? 1 : 0)) * L::kRows;
        for (int r = threadIdx.x; r < n_rows; r += W * 32) {
            float2 v[W];
            float best = -INFINITY, sum = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                v[w] = ld_shared_f32x2(ml_s + (w * L::kRows + r) * 8);
                best = fmaxf(best, v[w].x);
            }
            const float use = best == -INFINITY ? 0.f : best;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float f = exp2_fast(v[w].x - use);
                sum += v[w].y * f;
                st_shared_f32(ml_s + (w * L::kRows + r) * 8, f);
            }
            st_shared_f32(row_s + r * 4, whole ? (sum == 0.f ? 0.f : (FP8 ? 1.f / kF16Head : 1.f) / sum) : 1.f);
            if (!whole) {
                if (p.join) st_shared_f32x2(join_s + L::kRows * D * 4 + r * 8, best, sum);
                else p.part_ml[piece_row + r] = make_float2(best, sum);
            } else if (a.lse) {
                const int step = r / a.group, h = r - step * a.group;
                a.lse[(static_cast<int64_t>(s.b) * a.n_step + step) * a.H + head * a.group + h] =
                    sum == 0.f ? -INFINITY : (best + log2f(sum)) * 0.6931471805599453f;
            }
        }
        consumers_sync<W>();
        float f[NR][2];
#pragma unroll
        for (int nr = 0; nr < NR; ++nr)
#pragma unroll
            for (int e = 0; e < 2; ++e) f[nr][e] = ld_shared_f32(ml_s + (warp * L::kRows + nr * 8 + 2 * j + e) * 8);
#pragma unroll
        for (int c0 = 0; c0 < D; c0 += L::kSlice) {
#pragma unroll
            for (int nr = 0; nr < NR; ++nr)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t row = red_s + ((warp * L::kRows + nr * 8 + 2 * j + e) * L::kPitch) * 4;
#pragma unroll
                    for (int n0 = 0; n0 < L::kSlice / 16; ++n0) {
                        const float lo = o[nr][c0 / 16 + n0][e] * f[nr][e], hi = o[nr][c0 / 16 + n0][2 + e] * f[nr][e];
                        if (FP8) {               // columns 16 n + 2 g, + 1
                            st_shared_f32x2(row + (n0 * 16 + 2 * g) * 4, lo, hi);
                        } else {                 // 16 n + g, + 8
                            st_shared_f32(row + (n0 * 16 + g) * 4, lo);
                            st_shared_f32(row + (n0 * 16 + 8 + g) * 4, hi);
                        }
                    }
                }
            consumers_sync<W>();
            for (int i = threadIdx.x; i < n_rows * (L::kSlice / 4); i += W * 32) {
                const int r = i / (L::kSlice / 4), c = i % (L::kSlice / 4) * 4;
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    const float4 z = ld_shared_f32x4(red_s + ((w * L::kRows + r) * L::kPitch + c) * 4);
                    v.x += z.x;
                    v.y += z.y;
                    v.z += z.z;
                    v.w += z.w;
                }
                if (!whole) {
                    if (p.join) st_shared_v4(join_s + (r * D + c0 + c) * 4, make_uint4(__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w)));
                    else *reinterpret_cast<float4*>(p.part_o + (piece_row + r) * D + c0 + c) = v;
                } else {
                    const float over = ld_shared_f32(row_s + r * 4);
                    const int step = r / a.group, h = r - step * a.group;
                    const int64_t to = ((static_cast<int64_t>(s.b) * a.n_step + step) * a.H + head * a.group + h) * D + c0 + c;
                    *reinterpret_cast<uint2*>(a.out + to) = make_uint2(pack_bf16(v.x * over, v.y * over), pack_bf16(v.z * over, v.w * over));
                }
            }
            consumers_sync<W>();
        }
        if (p.join > 1) {
            // The cluster's parts: every CTA joins some of the rows, D / 2 threads each.
            cluster_sync();
            constexpr int T = D / 2;
            const int rank = blockIdx.x % p.join, c = threadIdx.x % T * 2;
            for (int r = rank + p.join * static_cast<int>(threadIdx.x / T); r < n_rows; r += p.join * (W * 32 / T)) {
                float2 ml[8], of[8];
                float best = -INFINITY;
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k < p.join) {
                        const uint32_t at = map_to_cta(join_s, k);
                        ml[k] = ld_cluster_f32x2(at + L::kRows * D * 4 + r * 8);
                        of[k] = ld_cluster_f32x2(at + (r * D + c) * 4);
                        best = fmaxf(best, ml[k].x);
                    }
                const float use = best == -INFINITY ? 0.f : best;
                float sum = 0.f, x = 0.f, y = 0.f;
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k < p.join) {
                        const float w = exp2_fast(ml[k].x - use);
                        sum += ml[k].y * w;
                        x += of[k].x * w;
                        y += of[k].y * w;
                    }
                const float over = sum == 0.f ? 0.f : (FP8 ? 1.f / kF16Head : 1.f) / sum;
                const int step = r / a.group, h = r - step * a.group;
                const int64_t row = (static_cast<int64_t>(s.b) * a.n_step + step) * a.H + head * a.group + h;
                *reinterpret_cast<uint32_t*>(a.out + row * D + c) = pack_bf16(x * over, y * over);
                if (a.lse && c == 0) a.lse[row] = sum == 0.f ? -INFINITY : (best + log2f(sum)) * 0.6931471805599453f;
            }
            cluster_sync();
            return;
        }
        if (s.t0 == 0 && !whole) owner = make_int4(s.b, s.head, pieces_of(run, s, p.heads), 0);
    }
    if (p.join) return;
    if (threadIdx.x == 0) p.owners[blockIdx.x] = owner;

    // Requests without keys: zeros and -inf.
    for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
        if (tiles_of(p, b) != 0) continue;
        const int64_t n_vec = static_cast<int64_t>(a.n_step) * a.H * (D / 8);
        uint4* to = reinterpret_cast<uint4*>(a.out + static_cast<int64_t>(b) * a.n_step * a.H * D);
        for (int64_t i = threadIdx.x; i < n_vec; i += W * 32) to[i] = make_uint4(0u, 0u, 0u, 0u);
        if (a.lse)
            for (int i = threadIdx.x; i < a.n_step * a.H; i += W * 32) a.lse[static_cast<int64_t>(b) * a.n_step * a.H + i] = -INFINITY;
    }
}

int max_grid(int cta_rows) { return cta_rows <= 8 ? 3 * kPagedMaxSms : (cta_rows <= 32 ? 2 * kPagedMaxSms : kPagedMaxSms); }
// of a block of rows: here up to 32, in paged_attn_rows.cu 128 or 256
int rows_of_cta(int rows) { return rows <= 8 ? 8 : (rows <= 16 ? 16 : (rows <= 32 ? 32 : (rows <= 128 ? 128 : 256))); }

template <int D, bool FP8, int NR>
cudaError_t run(const CUtensorMap& k_map, const CUtensorMap& v_map, Params& p, int sm_count, cudaStream_t stream, int* launches) {
    using L = Layout<D, FP8, NR>;
    // Heads in step: all of up to 8, else the largest divisor of their number up to 8.
    p.heads = p.a.c.H_kv < 8 ? p.a.c.H_kv : 8;
    while (p.a.c.H_kv % p.heads) --p.heads;
    p.units = p.a.c.H_kv / p.heads;
    p.tile_log2 = L::kTile == 64 ? 6 : 7;
    auto kernel = paged_attn_kernel<D, FP8, NR>;
    cudaError_t e = ensure_max_dynamic_smem(reinterpret_cast<const void*>(kernel), L::kBytes);
    if (e != cudaSuccess) return e;
    // Few units of few tiles: a unit a cluster, cut among as many CTAs (8 at most) as all have room at once, which join their parts over distributed
    // shared memory. One launch, and no scan over the requests; but every unit is cut alike, whatever its length, so only where that is at most
    // kJoinTiles tiles a CTA, or where the units are alike (selections) and a CTA has hardly more than an equal share of all tiles.
    const int64_t units = static_cast<int64_t>(p.a.B) * p.a.c.H_kv;
    int64_t keys = p.a.max_len;
    if (p.a.pages) {
        const int64_t pages = (keys + p.a.c.page_size - 1) / p.a.c.page_size;
        keys = (pages < p.a.n_sel ? pages : p.a.n_sel) * p.a.c.page_size;
    }
    const int64_t tiles = (keys + L::kTile - 1) / L::kTile;
    int join = 8;
    while (join > 1 && (units * join > sm_count * L::kCtas || join / 2 >= tiles)) join /= 2;
    const int64_t room = sm_count * L::kCtas;
    const bool alike = p.a.pages && tiles <= join * (units * tiles / room + kJoinSlack);
    p.join = units * join <= room && (tiles <= join * kJoinTiles || alike) ? join : 0;
    *launches += 1;
    if (p.join) {
        cudaLaunchAttribute attr[2]{};
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = static_cast<unsigned>(join);
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3(static_cast<unsigned>(units * join));
        cfg.blockDim = dim3(L::kThreads);
        cfg.dynamicSmemBytes = L::kBytes;
        cfg.stream = stream;
        cfg.attrs = attr;
        cfg.numAttrs = 2;
        return cudaLaunchKernelEx(&cfg, kernel, k_map, v_map, p);
    }
    const int most = sm_count * L::kCtas < max_grid(L::kRows) ? sm_count * L::kCtas : max_grid(L::kRows);
    const int grid = most / p.heads * p.heads;
    e = launch_behind(kernel, dim3(grid), L::kThreads, L::kBytes, stream, k_map, v_map, p);
    if (e != cudaSuccess) return e;
    const int rows = p.a.n_step * p.a.group < L::kRows ? p.a.n_step * p.a.group : L::kRows;
    *launches += 1;
    const float out_scale = FP8 ? 1.f / kF16Head : 1.f;
    if (grid / p.heads > 12 * static_cast<int64_t>(p.a.B) * p.units)       // runs per unit, and so pieces: more than a warp's three batches in flight
        return launch_behind(paged_merge_kernel<D, L::kRows, 4, 2>, dim3(grid, (rows + 1) / 2), 256, 0, stream, p, out_scale);
    return launch_behind(paged_merge_kernel<D, L::kRows, 1, 4>, dim3(grid, (rows + 3) / 4), 128, 0, stream, p, out_scale);
}

}  // namespace

// owners, the pieces' maxima and sums, the pieces
size_t paged_attn_workspace_bytes(int n_step, int group, int d) {
    const size_t rows = static_cast<size_t>(rows_of_cta(n_step * group)), grid = static_cast<size_t>(max_grid(static_cast<int>(rows)));
    return grid * 16 + grid * 2 * rows * (8 + static_cast<size_t>(d) * 4);
}
bool paged_attn_fits(const PagedAttnArgs& a) {
    const int64_t rows = static_cast<int64_t>(a.n_step) * a.group, cta = rows_of_cta(a.n_step * a.group);
    constexpr int kTile = 64;                    // (of the smallest tiles)
    int64_t keys = a.max_len + kTile;
    if (a.pages) {
        const int64_t pages = (a.max_len + a.c.page_size - 1) / a.c.page_size;
        keys = (pages < a.n_sel ? pages : a.n_sel) * a.c.page_size + kTile;
    }
    return static_cast<double>(a.B) * a.c.H_kv * ((rows + cta - 1) / cta) * (keys / kTile + kSegmentTiles) < 2147483648.0;
}

cudaError_t launch_paged_attn(const PagedAttnArgs& a, void* workspace, const CUtensorMap& k_map, const CUtensorMap& v_map, unsigned int* status,
                              int sm_count, cudaStream_t stream, int* launches) {
    if (a.n_step * a.group > kRowsHere) return launch_paged_attn_rows(a, workspace, k_map, v_map, status, sm_count, stream, launches);
    Params p{};
    p.a = a;
    const int cta_rows = rows_of_cta(a.n_step * a.group);
    p.row_blocks = 1;
    p.piece_log2 = a.c.page_size % 64 == 0 ? 6 : (a.c.page_size % 32 == 0 ? 5 : 4);
    p.scale_log2 = a.scale * 1.4426950408889634f;
    uint8_t* w = static_cast<uint8_t*>(workspace);
    p.owners = reinterpret_cast<int4*>(w);
    const size_t grid = static_cast<size_t>(max_grid(cta_rows));
    p.part_ml = reinterpret_cast<float2*>(w + grid * 16);
    p.part_o = reinterpret_cast<float*>(w + grid * 16 + grid * 2 * cta_rows * 8);
    p.status = status;
#define IDXC_RUN(D_, F_)                                                                                \
    (cta_rows == 8    ? run<D_, F_, 1>(k_map, v_map, p, sm_count, stream, launches)                      \
     : cta_rows == 16 ? run<D_, F_, 2>(k_map, v_map, p, sm_count, stream, launches)                      \
                      : run<D_, F_, 4>(k_map, v_map, p, sm_count, stream, launches))
    if (a.c.d == 128) return a.c.fp8 ? IDXC_RUN(128, true) : IDXC_RUN(128, false);
    return a.c.fp8 ? IDXC_RUN(64, true) : IDXC_RUN(64, false);
#undef IDXC_RUN
}

}  // namespace idxc
