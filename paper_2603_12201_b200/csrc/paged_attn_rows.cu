// Attention over a paged cache for many query rows a key head: prompts that go into the cache in chunks, many drafted tokens, large groups of heads.
//     x[s] = scale <q, k_s> over the visible keys s,   out = sum_s softmax(x)[s] v_s,   lse = log sum_s exp(x[s])
//
// What bounds it: with R rows a key and a value of d bf16 columns are 4 d bytes and 4 d R flops, R flops a byte: above 250 rows the tensor cores, and beside
// them the exponentials (16 a cycle and SM, as long as the two products of their 128 columns). So this is one CTA an SM on tcgen05: blocks of 128 rows, two of
// them (ways) for more than 128 rows, share every tile of 128 keys.
//     S = Q K^T      operands in shared memory, fp32 scores in tensor memory
//     O += P V       P as bf16 in tensor memory in place of its scores, V's rows as they lie (keys along the product's inner axis)
// A warpgroup a way turns scores into probabilities, a thread a row, so that maxima and sums need no other thread. While it does, the tensor cores work for
// the other way; one warp issues everything in the order PV(t - 1), S(t) of way 0, then of way 1, so that scores arriving mean that the output is at rest.
// A row's reference moves, and the output with it, only when a score passes it by 2^8.
//
// Measured (graph replays, one B200; 8 requests, 8 key heads, bf16, d = 128 / 64): 128 rows over 32768 keys 242 / 212 us (477 / 347 by paged_attn.cu's kernel), 512
// over 8192 183 / 151 (492 / 358), 4096 over 8192 1105 to 1210 / 957 (3760 / 2695): up to 996 / 574 TFLOP/s, with d = 64 twice the exponentials a flop.
//
// A warp fills a ring of tiles, K and V in turn, by TMA from pages or 16- to 64-key pieces of them. Runs of equal cost over all units (request, key head, block
// of rows), where a unit has the tiles that its last row sees; segments that runs cut go through the merge.
#include <cuda_bf16.h>

#include "kernels.h"
#include "paged_attn.cuh"
#include "ptx_sm100.cuh"

namespace idxc {
using namespace paged;
namespace {

constexpr int kTile = 128;                       // keys
constexpr int kWayRows = 128;
constexpr float kSlack = 8.f;                    // log2 units by which a score may pass its row's reference
constexpr int kSoftmaxWarps = 8, kThreads = (kSoftmaxWarps + 4) * 32;      // with the producer's, the products' and two idle warps
// A softmax thread holds a row's 128 scores: of the launch's 168 registers a thread the third warpgroup keeps 80.
constexpr int kOtherRegs = 80, kSoftmaxRegs = 208;
static_assert(128 * kOtherRegs + 256 * kSoftmaxRegs <= kThreads * 168, "shares of the launch's registers");
constexpr int kPosTiles = 8;                     // tiles whose positions are kept: more than the ring holds and the softmax works on

template <int D>
struct Layout {
    static constexpr int kBlock = kTile * 128;                         // bytes of 64 columns of a tile: rows of 128 bytes
    static constexpr int kSlotBytes = D / 64 * kBlock;
    static constexpr int kSlots = D == 128 ? 5 : 8;
    static constexpr int kQBytes = 2 * kWayRows * D * 2;
    static constexpr int kSmall = 1024;
    static constexpr int kBytes = 1024 + kSlots * kSlotBytes + kQBytes + kSmall;
    static constexpr uint32_t kColO = 256;                             // tensor memory: scores of way w at 128 w, output at kColO + D w
    static_assert(kBytes <= 232448, "shared memory of a CTA");
    static_assert(kSlots * 16 + 8 * 8 + kPosTiles * 32 + 128 <= kSmall, "small words");
};

// Tiles of block r of a request's rows: of the keys that its last row sees, or of the selection.
__device__ __forceinline__ int tiles_of_block(const Params& p, int b, int r) {
    if (p.a.pages) return tiles_of(p, b);
    const int block = p.ways * kWayRows, last = min((r * block + block - 1) / p.a.group, p.a.n_step - 1);
    return (max(length_of(p.a, b) - (p.a.n_step - 1 - last), 0) + kTile - 1) / kTile;
}
__device__ __forceinline__ int length_of_head(const Params& p, int b) {
    int n = 0;
    for (int r = 0; r < p.row_blocks; ++r) n += length_of_unit(tiles_of_block(p, b, r));
    return n;
}
struct Walk {
    const Params& p;
    int b, head, r, x, left;
    __device__ __forceinline__ Walk(const Params& q, const Run& run) : p(q), b(run.b), head(0), r(0), x(run.x), left(run.n) {
        if (left == 0) return;
        const int per_head = length_of_head(p, b);
        head = x / per_head;
        x -= head * per_head;
    }
    __device__ __forceinline__ bool next(Segment& s) {
        while (left > 0 && b < p.a.B) {
            const int nt = tiles_of_block(p, b, r), len = length_of_unit(nt);
            if (x >= len) {
                x -= len;
                if (++r == p.row_blocks) {
                    r = 0;
                    if (++head == p.a.c.H_kv) {
                        head = 0;
                        ++b;
                    }
                }
                continue;
            }
            const int n = min(len - x, left);
            s.b = b;
            s.head = head;
            s.rows = r;
            s.nt = nt;
            s.t0 = max(x - kSegmentTiles, 0);
            s.n = max(x + n - kSegmentTiles, 0) - s.t0;
            x += n;
            left -= n;
            if (s.n > 0) return true;
        }
        return false;
    }
};

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
paged_rows_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const __grid_constant__ Params p) {
    using L = Layout<D>;
    constexpr int NS = L::kSlots;
    extern __shared__ uint8_t raw[];
    const uint32_t base = smem_u32(raw);
    const uint32_t slots = (base + 1023u) & ~1023u;
    const uint32_t q_s = slots + NS * L::kSlotBytes;
    const uint32_t bar_full = q_s + L::kQBytes, bar_empty = bar_full + NS * 8;
    const uint32_t bar_q = bar_empty + NS * 8, bar_s = bar_q + 16, bar_p = bar_s + 16, bar_o = bar_p + 16;      // of two ways each
    const uint32_t pos_s = bar_o + 16;           // [kPosTiles][8] position of the first key of each piece, -1: none
    const uint32_t tmem_s = pos_s + kPosTiles * 32, flag_s = tmem_s + 4, scratch_s = flag_s + 4;
    volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(raw + (flag_s - base));
    int* scratch = reinterpret_cast<int*>(raw + (scratch_s - base));

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < NS; ++i) {
            mbar_init(bar_full + 8 * i, 1);
            mbar_init(bar_empty + 8 * i, 1);
        }
        for (int w = 0; w < 2; ++w) {
            mbar_init(bar_q + 8 * w, kWayRows);
            mbar_init(bar_s + 8 * w, 1);
            mbar_init(bar_p + 8 * w, 4);
            mbar_init(bar_o + 8 * w, 1);
        }
        *abort_flag = 0;
        fence_mbar_init();
        tma_prefetch_desc(&k_map);
        tma_prefetch_desc(&v_map);
    }
    if (warp == kSoftmaxWarps + 1) {
        tmem_alloc(tmem_s, 512);
        tmem_relinquish_alloc_permit();
        tcgen05_fence_before_sync();
    }
    let_next_start();
    wait_for_previous();
    const PagedAttnArgs& a = p.a;
    const int H_kv = a.c.H_kv;
    const Run run = find_run(p, scratch, [&](int b) { return length_of_head(p, b) * H_kv; });      // (its barriers publish the mbarriers and tensor memory's place too)
    tcgen05_fence_after_sync();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(raw + (tmem_s - base));
    const int rows_all = a.n_step * a.group, block_rows = p.ways * kWayRows;
    auto ways_of = [&](const Segment& s) { return rows_all - s.rows * block_rows > kWayRows ? 2 : 1; };
    auto give_up = [&](unsigned code) {
        if (lane == 0) {
            *abort_flag = 1;
            atomicCAS(p.status, DEV_OK, code);
        }
    };

    if (warp < kSoftmaxWarps) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        // ------------------------------------------------------------ softmax: a thread a row
        const int w = warp >> 2, tid = threadIdx.x & 127;
        const uint32_t lanes = static_cast<uint32_t>(warp & 3) * 32u << 16;
        const uint32_t s_col = tmem + 128 * w + lanes, o_col = tmem + L::kColO + D * w + lanes;
        const int per_tile = kTile >> p.piece_log2, piece = 1 << p.piece_log2;
        uint32_t n_s = 0, n_o = 0;
        int it = 0;
        bool ok = true;
        int4 owner = make_int4(-1, 0, 0, 0);
        auto wait = [&](uint32_t bar, uint32_t parity) {
            if (ok && !mbar_wait(bar, parity, abort_flag)) ok = false;
            ok = __all_sync(0xFFFFFFFFu, ok);
            return ok;
        };
        Walk walk(p, run);
        Segment s;
        while (ok && walk.next(s)) {
            const bool whole = s.t0 == 0 && s.n == s.nt;
            if (s.t0 == 0 && !whole) owner = make_int4(s.b, s.head * p.row_blocks + s.rows, pieces_of(run, s, 1), 0);
            if (w >= ways_of(s)) {
                it += s.n;
                continue;
            }
            const int len = length_of(a, s.b), row0 = s.rows * block_rows + w * kWayRows;
            // ---- q, whose last readers were the products behind the output that this warpgroup has seen
#pragma unroll 8
            for (int i = tid; i < kWayRows * (D / 8); i += 128) {
                const int r = i / (D / 8), c = i % (D / 8);
                uint4 q = make_uint4(0u, 0u, 0u, 0u);
                if (row0 + r < rows_all) {
                    const int step = (row0 + r) / a.group, h = row0 + r - step * a.group;
                    q = reinterpret_cast<const uint4*>(a.q + (static_cast<int64_t>(s.b) * a.n_step + step) * a.q_stride +
                                                       static_cast<int64_t>(s.head * a.group + h) * D)[c];
                }
                st_shared_v4(q_s + (w * (D / 64) + (c >> 3)) * (kWayRows * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4), q);
            }
            fence_proxy_async_smem();
            mbar_arrive(bar_q + 8 * w);

            const int row = row0 + tid, step = min(row / a.group, a.n_step - 1);
            const int sees = len - (a.n_step - 1 - step), sees_least = len - (a.n_step - 1 - row0 / a.group);
            float m = -INFINITY, l = 0.f;
            for (int t = 0; t < s.n; ++t) {
                const int vi = 2 * (it + t) + 1, v_slot = vi % NS;
                const uint32_t pos_at = pos_s + ((it + t) % kPosTiles) * 32;
                // Scores first: a way that had no rows in a segment before this one would take an older phase of the slot's barrier for its own. V's arrival
                // publishes the positions; the slot's next copy waits for this tile's probabilities.
                if (!wait(bar_s + 8 * w, n_s++ & 1) || !wait(bar_full + 8 * v_slot, (vi / NS) & 1)) break;
                tcgen05_fence_after_sync();
                int pos = 0;
                if (lane < per_tile) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(pos) : "r"(pos_at + lane * 4) : "memory");
                const bool clean = __all_sync(0xFFFFFFFFu, lane >= per_tile || (pos >= 0 && pos + piece <= sees_least));
                if (w == 0 && !clean) {
                    // rows of V that no token sees meet probability 0 and may hold anything: they are cleared, way 1's too, whose product follows way 0's
                    const int first = __shfl_sync(0xFFFFFFFFu, pos, tid >> p.piece_log2);
                    if (first < 0 || first + (tid & (piece - 1)) >= len) {
#pragma unroll
                        for (int c = 0; c < D / 8; ++c)
                            st_shared_v4(slots + v_slot * L::kSlotBytes + (c >> 3) * L::kBlock + tid * 128 + ((c & 7) << 4), make_uint4(0u, 0u, 0u, 0u));
                        fence_proxy_async_smem();
                    }
                }
                uint32_t x[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld_32x32b_x32(s_col + 32 * c, x[c]);
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld_wait(x[c]);
                float scale = p.scale_log2;
                if (!clean || !(scale > 0.f)) {
#pragma unroll
                    for (int g = 0; g < 8; ++g) {                             // 16 keys
                        const int first = __shfl_sync(0xFFFFFFFFu, pos, g * 16 >> p.piece_log2);
                        const int n = first < 0 ? 0 : sees - first - (g * 16 & (piece - 1));
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            uint32_t& y = x[g / 2][g % 2 * 16 + e];
                            y = __float_as_uint(e < n ? __uint_as_float(y) * scale : -INFINITY);
                        }
                    }
                    scale = 1.f;
                }
                float top4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int e = 0; e < 32; ++e) top4[e & 3] = fmaxf(top4[e & 3], __uint_as_float(x[c][e]));
                const float top = fmaxf(fmaxf(top4[0], top4[1]), fmaxf(top4[2], top4[3])) * scale;
                if (__any_sync(0xFFFFFFFFu, !(top <= m + kSlack))) {
                    const float v = fmaxf(m, top), f = exp2_fast(m - (v == -INFINITY ? 0.f : v));
                    m = v;
                    l *= f;
                    if (t > 0) {                                              // the scores are there, so the products before them are done
#pragma unroll 1
                        for (int c = 0; c < D; c += 32) {
                            uint32_t o[32];
                            tmem_ld_32x32b_x32(o_col + c, o);
                            tmem_ld_wait(o);
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                            tmem_st_32x32b_x32(o_col + c, o);
                        }
                    }
                }
                const float use = m == -INFINITY ? 0.f : m;
                float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < 8; ++c) {                                 // 16 keys
                    uint32_t y[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float p0 = exp2_fast(fmaf(__uint_as_float(x[c / 2][c % 2 * 16 + 2 * e]), scale, -use));
                        const float p1 = exp2_fast(fmaf(__uint_as_float(x[c / 2][c % 2 * 16 + 2 * e + 1]), scale, -use));
                        sum[2 * (e & 1)] += p0;
                        sum[2 * (e & 1) + 1] += p1;
                        y[e] = pack_bf16(p0, p1);
                    }
                    tmem_st_32x32b_x8(s_col + 8 * c, y);
                }
                l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
                tmem_st_wait();
                tcgen05_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_p + 8 * w);
            }
            it += s.n;
            if (!wait(bar_o + 8 * w, n_o++ & 1)) break;
            tcgen05_fence_after_sync();
            // ---- output
            const bool writes = row < rows_all;
            const int64_t out_row = (static_cast<int64_t>(s.b) * a.n_step + step) * a.H + s.head * a.group + (row - step * a.group);
            const int64_t piece_row = (static_cast<int64_t>(blockIdx.x) * 2 + (s.t0 == 0 ? 1 : 0)) * block_rows + w * kWayRows + tid;
            const float over = !whole ? 1.f : (l == 0.f ? 0.f : 1.f / l);
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
                uint32_t o[32];
                tmem_ld_32x32b_x32(o_col + c, o);
                tmem_ld_wait(o);
                if (!writes) continue;
                if (whole) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint32_t v[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) v[k] = pack_bf16(__uint_as_float(o[8 * e + 2 * k]) * over, __uint_as_float(o[8 * e + 2 * k + 1]) * over);
                        reinterpret_cast<uint4*>(a.out + out_row * D + c)[e] = make_uint4(v[0], v[1], v[2], v[3]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        reinterpret_cast<uint4*>(p.part_o + piece_row * D + c)[e] = make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                }
            }
            tcgen05_fence_before_sync();         // (the next segment's first product follows this thread's next arrival)
            if (writes) {
                if (!whole) p.part_ml[piece_row] = make_float2(m, l);
                else if (a.lse) a.lse[out_row] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
            }
        }
        if (!ok) give_up(DEV_TIMEOUT_EPILOGUE);
        if (threadIdx.x == 0) p.owners[blockIdx.x] = owner;
        // Blocks of rows that see no key: zeros and -inf.
        const int blocks = H_kv * p.row_blocks;
        for (int64_t u = blockIdx.x; u < static_cast<int64_t>(a.B) * blocks; u += gridDim.x) {
            const int b = static_cast<int>(u / blocks), of = static_cast<int>(u - static_cast<int64_t>(b) * blocks), head = of / p.row_blocks, r = of - head * p.row_blocks;
            if (tiles_of_block(p, b, r) != 0) continue;
            for (int i = threadIdx.x; i < block_rows * (D / 8); i += kSoftmaxWarps * 32) {
                const int row = r * block_rows + i / (D / 8);
                if (row >= rows_all) break;
                const int step = row / a.group;
                const int64_t to = (static_cast<int64_t>(b) * a.n_step + step) * a.H + head * a.group + (row - step * a.group);
                reinterpret_cast<uint4*>(a.out + to * D)[i % (D / 8)] = make_uint4(0u, 0u, 0u, 0u);
                if (a.lse && i % (D / 8) == 0) a.lse[to] = -INFINITY;
            }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        if (warp == kSoftmaxWarps) {
            // ------------------------------------------------------------ producer: K and V of a tile into the next two slots of the ring
            const int piece = 1 << p.piece_log2, per_tile_log2 = 7 - p.piece_log2, per_tile = 1 << per_tile_log2;
            const uint32_t piece_bytes = static_cast<uint32_t>(piece) * D * 2;
            const int P = a.c.page_size;
            int it = 0;                              // tiles
            bool ok = true;
            Walk walk(p, run);
            Segment s;
            while (ok && walk.next(s)) {
                const int len = length_of(a, s.b);
                const int32_t* table = a.table + static_cast<int64_t>(s.b) * a.ld_table;
                const int32_t* sel = a.pages ? a.pages + (static_cast<int64_t>(s.b) * H_kv + s.head) * a.n_sel : nullptr;
                const int n_entries = (len + P - 1) / P, most = sel ? min(a.n_sel, n_entries) : n_entries;
                const int n_pieces = s.n << per_tile_log2;
                struct Where { int page, off, pos; };
                auto locate = [&](int i) -> Where {
                    Where w{0, 0, -1};
                    if (i < n_pieces) {
                        const unsigned v = static_cast<unsigned>(s.t0) * kTile + (static_cast<unsigned>(i) << p.piece_log2);
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
                for (int i0 = 0; ok && i0 < n_pieces; i0 += 32) {
                    const Where now = next;
                    if (i0 + 32 < n_pieces) next = locate(i0 + 32 + lane);
                    const int n_here = min(32, n_pieces - i0) >> per_tile_log2;      // tiles
                    for (int t = 0; t < n_here; ++t, ++it) {
                        const bool mine = (lane >> per_tile_log2) == t;
                        const int in_tile = lane & (per_tile - 1);
                        const uint32_t bytes = __popc(__ballot_sync(0xFFFFFFFFu, mine && now.pos >= 0)) * piece_bytes;
#pragma unroll
                        for (int kv = 0; kv < 2; ++kv) {
                            const int i = 2 * it + kv, slot = i % NS;
                            if (ok && i >= NS && !mbar_wait(bar_empty + 8 * slot, ((i / NS) & 1) ^ 1, abort_flag)) {
                                give_up(DEV_TIMEOUT_PRODUCER);
                                ok = false;
                            }
                            ok = __all_sync(0xFFFFFFFFu, ok);
                            if (!ok) break;
                            if (kv == 0 && mine)
                                asm volatile("st.shared.b32 [%0], %1;" ::"r"(pos_s + (it % kPosTiles) * 32 + in_tile * 4), "r"(now.pos) : "memory");
                            __syncwarp();
                            const uint32_t full = bar_full + 8 * slot;
                            if (lane == 0) mbar_arrive_expect_tx(full, bytes);
                            __syncwarp();
                            if (mine && now.pos >= 0) {
                                const uint32_t to = slots + slot * L::kSlotBytes + in_tile * piece * 128;
#pragma unroll
                                for (int h = 0; h < D / 64; ++h) tma_load_4d(to + h * L::kBlock, kv ? &v_map : &k_map, full, h * 64, now.off, s.head, now.page);
                            }
                        }
                        if (!ok) break;
                    }
                }
            }
        } else if (warp == kSoftmaxWarps + 1) {
            // ------------------------------------------------------------ products
            constexpr uint32_t kIdescS = umma_idesc(1, 1, 128, kTile), kIdescO = umma_idesc(1, 1, 128, D) | kUmmaBMajorMN;
            uint32_t n_q[2] = {0u, 0u}, n_p[2] = {0u, 0u};
            int it = 0;
            bool ok = true;
            auto wait = [&](uint32_t bar, uint32_t parity) {
                if (ok && !mbar_wait(bar, parity, abort_flag)) ok = false;
                ok = __all_sync(0xFFFFFFFFu, ok);
                tcgen05_fence_after_sync();
                return ok;
            };
            Walk walk(p, run);
            Segment s;
            while (ok && walk.next(s)) {
                const int ways = ways_of(s);
                for (int t = 0; ok && t <= s.n; ++t) {
                    const int ki = 2 * (it + t), vi = ki - 1, k_slot = ki % NS, v_slot = (vi + NS) % NS;
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        if (w >= ways) break;
                        if (t > 0) {
                            if (!wait(bar_p + 8 * w, n_p[w]++ & 1)) break;
                            if (w == 0 && !wait(bar_full + 8 * v_slot, (vi / NS) & 1)) break;
                            const uint64_t v_desc = umma_smem_desc_sw128_mn(slots + v_slot * L::kSlotBytes, L::kBlock);
#pragma unroll
                            for (int k = 0; k < kTile / 16; ++k)
                                umma_f16_ts_elect_acc(tmem + L::kColO + D * w, tmem + 128 * w + 8 * k, v_desc + k * 128, kIdescO, t > 1 || k > 0);
                            if (w == ways - 1) umma_commit_elect(bar_empty + 8 * v_slot);
                            if (t == s.n) umma_commit_elect(bar_o + 8 * w);
                        }
                        if (t < s.n) {
                            if (t == 0 && !wait(bar_q + 8 * w, n_q[w]++ & 1)) break;
                            if (w == 0 && !wait(bar_full + 8 * k_slot, (ki / NS) & 1)) break;
#pragma unroll
                            for (int h = 0; h < D / 64; ++h)
                                umma_f16_x4<2, 2>(tmem + 128 * w, umma_smem_desc_sw128(q_s + (w * (D / 64) + h) * kWayRows * 128),
                                                  umma_smem_desc_sw128(slots + k_slot * L::kSlotBytes + h * L::kBlock), kIdescS, h > 0);
                            umma_commit_elect(bar_s + 8 * w);
                            if (w == ways - 1) umma_commit_elect(bar_empty + 8 * k_slot);
                        }
                    }
                }
                it += s.n;
            }
            if (!ok) give_up(DEV_TIMEOUT_MMA);
        }
    }

    // ---------------------------------------------------------------- teardown
    __syncwarp();
    if (*abort_flag) {                           // copies may still be in flight: let them land before the CTA's memory goes
        const long long t0 = clock64();
        while (clock64() - t0 < 2000000LL) __nanosleep(1000);
    }
    tcgen05_fence_before_sync();
    __syncthreads();
    if (warp == kSoftmaxWarps + 1) {
        tcgen05_fence_after_sync();
        tmem_dealloc(tmem, 512);
    }
}

template <int D>
cudaError_t run_rows(const CUtensorMap& k_map, const CUtensorMap& v_map, const Params& p, int grid, cudaStream_t stream, int* launches) {
    cudaError_t e = ensure_max_dynamic_smem(reinterpret_cast<const void*>(paged_rows_kernel<D>), Layout<D>::kBytes);
    if (e != cudaSuccess) return e;
    *launches += 1;
    e = launch_behind(paged_rows_kernel<D>, dim3(grid), kThreads, Layout<D>::kBytes, stream, k_map, v_map, p);
    if (e != cudaSuccess) return e;
    const int rows = p.a.n_step * p.a.group < p.ways * kWayRows ? p.a.n_step * p.a.group : p.ways * kWayRows;
    *launches += 1;
    if (p.ways == 1) return launch_behind(paged_merge_kernel<D, kWayRows, 1, 4>, dim3(grid, (rows + 3) / 4), 128, 0, stream, p, 1.f);
    return launch_behind(paged_merge_kernel<D, 2 * kWayRows, 1, 4>, dim3(grid, (rows + 3) / 4), 128, 0, stream, p, 1.f);
}

}  // namespace

cudaError_t launch_paged_attn_rows(const PagedAttnArgs& a, void* workspace, const CUtensorMap& k_map, const CUtensorMap& v_map, unsigned int* status,
                                   int sm_count, cudaStream_t stream, int* launches) {
    Params p{};
    p.a = a;
    p.ways = a.n_step * a.group > kWayRows ? 2 : 1;
    const int block = p.ways * kWayRows;
    p.row_blocks = (a.n_step * a.group + block - 1) / block;
    p.heads = 1;
    p.tile_log2 = 7;
    p.piece_log2 = a.c.page_size % 64 == 0 ? 6 : (a.c.page_size % 32 == 0 ? 5 : 4);
    p.scale_log2 = a.scale * 1.4426950408889634f;
    p.status = status;
    const size_t most = kPagedMaxSms;
    uint8_t* w = static_cast<uint8_t*>(workspace);
    p.owners = reinterpret_cast<int4*>(w);
    p.part_ml = reinterpret_cast<float2*>(w + most * 16);
    p.part_o = reinterpret_cast<float*>(w + most * 16 + most * 2 * block * 8);
    const int grid = sm_count < kPagedMaxSms ? sm_count : kPagedMaxSms;
    return a.c.d == 128 ? run_rows<128>(k_map, v_map, p, grid, stream, launches) : run_rows<64>(k_map, v_map, p, grid, stream, launches);
}

}  // namespace idxc
