// Attention over a paged cache for many query rows a key head: prompts that go into the cache in chunks, many drafted tokens, large groups of heads.
//     x[s] = scale <q, k_s> over the visible keys s,   out = sum_s softmax(x)[s] v_s,   lse = log sum_s exp(x[s])
//
// What bounds it: with R rows a key and a value of d bf16 columns are 4 d bytes and 4 d R flops, R flops a byte: above 250 rows the tensor cores, and beside
// them the exponentials (16 a cycle and SM, as many cycles as the two products of their 128 columns take). So this is one CTA an SM on tcgen05:
//     S = Q K^T      128 rows by a tile of 128 keys, operands in shared memory, fp32 scores in tensor memory
//     O += P V       P as bf16 in tensor memory in place of its scores, V's rows as they lie (keys along the product's inner axis)
// Two ways, each with scores, an output and a warpgroup that turns scores into probabilities, a thread a row, so that maxima and sums need no other thread.
// While it does, the tensor cores work for the other way; one warp issues everything, PV of a way's tile before S of its next, so that scores arriving
// mean that the output is at rest. A row's reference moves, and the output with it, only when a score passes it by 2^8. More than 128 rows: each way has
// a block of 128 rows, and both share every tile. Fewer: both have the same rows and take tiles in turn, and their outputs meet in shared memory at the end
// (8 x 32768 keys, 8 key heads, 128 rows, d = 128 / 64: 196 / 137 us, 242 / 212 with one way). Up to 64 rows: the 128 rows are two copies, each with the
// probabilities of half of a tile's keys and zeros for the others, which halves a thread's share (64 rows 186 / 134 -> 183 / 111 us, 8 bits 273 / 210 -> 232 / 182).
//
// A warp fills a ring of tiles, K and V in turn, by TMA from pages or 16- to 64-key pieces of them. 8 bits: the ring holds codes, which four warps turn into f16
// (exact) in a second ring, with q as f16 times a power of two a row and the value's scale in the probability, whose reference is the running
// maximum of x + log2(scale), rounded up. Runs of equal cost over all units (request, key head, block of rows), where a unit has the tiles that its
// last row sees; segments that runs cut go through the merge.
//
// Measured (graph replays, one B200; 8 requests, 8 key heads, d = 128 / 64; in brackets with the warp-level instructions of paged_attn.cu, 8 warps a CTA):
//     rows   keys     bf16 us                   8 bits us
//       64  32768     183 / 111 (240 / 183)      232 / 182 (305 / 227)
//      128  32768     196 / 137 (477 / 347)      299 / 217 (540 / 424)
//      512   8192     171 / 147 (492 / 358)      276 / 236 (560 / 436)
//     4096   8192    1038 / 925 (3760 / 2695)   1770 / 1570 (4311 / 3322)
// so up to 1060 / 595 TFLOP/s in bf16 (d = 128: 945 to 1060 from run to run), 620 / 350 in 8 bits. A request's first 1024 tokens at once (8192 rows, half of
// the tiles): 317 / 254 us. What is left in bf16: with d = 64 the exponentials (twice as many a flop); in 8 bits the softmax threads' instructions, two
// products and a sum more a score, and up to 64 rows the four warps that convert.
// Tried: 208 and 80 registers come without spills only if each role's code begins with its own setmaxnreg (3142 us with scores spilled to local memory, 1105
// without); a thread's vectors of q loaded one after the other, and rows of the output written by their threads, 415 us for those first tokens.
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
constexpr int kSoftmaxWarps = 8, kProducerWarp = 8, kProductsWarp = 9, kConvertWarp = 10, kConvertWarps = 4;
constexpr int kPosTiles = 16, kScaleTiles = 8;   // tiles whose positions and scales are kept: more than the rings hold and the softmax works on

template <int D, bool FP8, int WAYS>
struct Layout {
    // bf16: two idle warps fill up the third warpgroup. 8 bits: the third and fourth are producer, products, four warps that convert, two idle ones.
    // A softmax thread holds a row's 128 scores, so registers go to it by warpgroups.
    static constexpr int kThreads = FP8 ? 512 : 384;
    static constexpr int kOtherRegs = FP8 ? 72 : 80, kSoftmaxRegs = FP8 ? 184 : 208;
    static_assert((kThreads - 256) * kOtherRegs + 256 * kSoftmaxRegs <= kThreads * (FP8 ? 128 : 168), "shares of the launch's registers");
    static constexpr int kBlock = kTile * 128;                         // bytes of 64 columns of a tile in 16 bits: rows of 128 bytes
    static constexpr int kSlotBytes = D / 64 * kBlock;
    static constexpr int kSlots = FP8 ? (D == 64 ? 6 : (WAYS == 1 ? 4 : 3)) : (D == 64 ? 8 : (WAYS == 1 ? 6 : 5));
    static constexpr int kRaws = FP8 ? (D == 64 ? 8 : 3) : 0;          // tiles of codes and scales
    static constexpr int kCodes = kTile * D;
    static constexpr int kRawBytes = FP8 ? kCodes + 1024 : 0;
    static constexpr int kQBytes = WAYS * kWayRows * D * 2;            // WAYS == 1: a quarter of both ways' outputs in fp32 as well
    static constexpr int kScaleBytes = FP8 ? kScaleTiles * 3 * kTile * 4 : 0;
    static constexpr int kPowerBytes = FP8 ? WAYS * kWayRows * 4 : 0;  // of two, taken out of a row of q
    static constexpr int kSmall = 1024;
    static constexpr int kBytes = 1024 + kSlots * kSlotBytes + kRaws * kRawBytes + kQBytes + kScaleBytes + kPowerBytes + kSmall;
    static constexpr uint32_t kColO = 256;                             // tensor memory: scores of way w at 128 w, output at kColO + D w
    static_assert(kBytes <= 232448, "shared memory of a CTA");
    static_assert((kSlots + kRaws) * 16 + 8 * 8 + kPosTiles * 32 + 128 <= kSmall, "small words");
};

__device__ __forceinline__ void threads_sync(int barrier, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(threads) : "memory"); }

__device__ __forceinline__ void tmem_ld_columns(uint32_t at, uint32_t (&o)[32]) { tmem_ld_32x32b_x32(at, o); }
__device__ __forceinline__ void tmem_ld_columns(uint32_t at, uint32_t (&o)[16]) { tmem_ld_32x32b_x16(at, o); }

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

template <int D, bool FP8, int WAYS, int R>
__global__ void __launch_bounds__((Layout<D, FP8, WAYS>::kThreads), 1)
paged_rows_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const __grid_constant__ Params p) {
    using L = Layout<D, FP8, WAYS>;
    constexpr int NS = L::kSlots, NR = FP8 ? L::kRaws : NS;            // tiles of 16-bit elements; what the producer fills
    constexpr int kBlockRows = WAYS == 1 ? R : 2 * kWayRows;
    constexpr int COPIES = kWayRows / R, NX = R / 32;                  // of the rows; a copy takes R of a tile's keys
    static_assert(WAYS == 1 || R == kWayRows, "copies with one block of rows only");
    constexpr float kHead = FP8 ? kF16Head : 1.f;
    extern __shared__ uint8_t raw[];
    const uint32_t base = smem_u32(raw);
    const uint32_t slots = (base + 1023u) & ~1023u;
    const uint32_t raws = FP8 ? slots + NS * L::kSlotBytes : slots;
    const uint32_t q_s = slots + NS * L::kSlotBytes + L::kRaws * L::kRawBytes;
    const uint32_t scale_s = q_s + L::kQBytes;   // [kScaleTiles][scales of K, log2 of V's, V's times 2^6][keys]
    const uint32_t row_s = scale_s + L::kScaleBytes;
    const uint32_t bar_full = row_s + L::kPowerBytes, bar_empty = bar_full + NS * 8;
    const uint32_t bar_raw = FP8 ? bar_empty + NS * 8 : bar_full, bar_raw_empty = FP8 ? bar_raw + NR * 8 : bar_empty;
    const uint32_t bar_q = bar_empty + NS * 8 + L::kRaws * 16, bar_s = bar_q + 16, bar_p = bar_s + 16, bar_o = bar_p + 16;      // of two ways each
    const uint32_t pos_s = bar_o + 16;           // [kPosTiles][8] position of the first key of each piece, -1: none
    const uint32_t tmem_s = pos_s + kPosTiles * 32, flag_s = tmem_s + 4, scratch_s = flag_s + 4;
    volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(raw + (flag_s - base));
    int* scratch = reinterpret_cast<int*>(raw + (scratch_s - base));

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < NS; ++i) {
            mbar_init(bar_full + 8 * i, FP8 ? kConvertWarps : 1);
            mbar_init(bar_empty + 8 * i, 1);
        }
        for (int i = 0; i < L::kRaws; ++i) {
            mbar_init(bar_raw + 8 * i, 1);
            mbar_init(bar_raw_empty + 8 * i, kConvertWarps);
        }
        for (int w = 0; w < 2; ++w) {
            mbar_init(bar_q + 8 * w, WAYS == 1 ? 256 : 128);
            mbar_init(bar_s + 8 * w, 1);
            mbar_init(bar_p + 8 * w, 4);
            mbar_init(bar_o + 8 * w, 1);
        }
        *abort_flag = 0;
        fence_mbar_init();
        if (p.a.c.n_pages > 0) {                 // (a cache without pages has no maps)
            tma_prefetch_desc(&k_map);
            tma_prefetch_desc(&v_map);
        }
    }
    if (warp == kProductsWarp) {
        tmem_alloc(tmem_s, 512);
        tmem_relinquish_alloc_permit();
        tcgen05_fence_before_sync();
    }
    let_next_start();
    wait_for_previous();
    const PagedAttnArgs& a = p.a;
    const int H_kv = a.c.H_kv;
    const Run run = find_run(p, scratch, [&](int b) { return length_of_head(p, b) * H_kv; });      // (its barriers publish what was set up here)
    tcgen05_fence_after_sync();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(raw + (tmem_s - base));
    const int rows_all = a.n_step * a.group;
    const int piece_log2 = p.piece_log2, piece = 1 << piece_log2, per_tile_log2 = 7 - piece_log2, per_tile = 1 << per_tile_log2;
    auto ways_of = [&](const Segment& s) { return rows_all - s.rows * kBlockRows > kWayRows ? 2 : 1; };      // (of WAYS == 2)
    auto give_up = [&](unsigned code) {
        if (lane == 0) atomicCAS(p.status, DEV_OK, code);
    };
    bool ok = true;                              // of a warp; one that has given up waits for nothing, but comes to every barrier of threads
    auto wait = [&](uint32_t bar, uint32_t parity) {
        if (ok && !mbar_wait(bar, parity, abort_flag)) {
            *abort_flag = 1;
            ok = false;
        }
        ok = __all_sync(0xFFFFFFFFu, ok);
        return ok;
    };

    if (warp < kSoftmaxWarps) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(L::kSoftmaxRegs));
        // ------------------------------------------------------------ softmax: a thread a row
        const int w = warp >> 2, tid = threadIdx.x & 127;
        const uint32_t lanes = static_cast<uint32_t>(warp & 3) * 32u << 16;
        const uint32_t s_col = tmem + 128 * w + lanes, o_col = tmem + L::kColO + D * w + lanes;
        const int q_block = WAYS == 1 ? 0 : w;
        uint32_t n_s = 0, n_o = 0;
        int it = 0;
        int4 owner = make_int4(-1, 0, 0, 0);
        Walk walk(p, run);
        Segment s;
        while (walk.next(s)) {
            const bool whole = s.t0 == 0 && s.n == s.nt;
            if (s.t0 == 0 && !whole) owner = make_int4(s.b, s.head * p.row_blocks + s.rows, pieces_of(run, s, 1), 0);
            if (WAYS == 2 && w >= ways_of(s)) {
                it += s.n;
                continue;
            }
            const int len = length_of(a, s.b), row0 = s.rows * kBlockRows + q_block * kWayRows;
            // ---- q, whose last readers were the products behind the outputs that have been seen. WAYS == 1: half of the rows by each warpgroup.
            constexpr int Q_THREADS = WAYS == 1 ? 256 : 128;
            constexpr int QV = kWayRows * (D / 8) / Q_THREADS;                // vectors of a thread, all on their way at a time
            uint4 q_v[QV];
#pragma unroll
            for (int u = 0; u < QV; ++u) {
                const int i = (WAYS == 1 ? threadIdx.x : tid) + u * Q_THREADS, r = i / (D / 8) % R, c = i % (D / 8);
                q_v[u] = make_uint4(0u, 0u, 0u, 0u);
                if (row0 + r < rows_all) {
                    const int step = (row0 + r) / a.group, h = row0 + r - step * a.group;
                    q_v[u] = reinterpret_cast<const uint4*>(a.q + (static_cast<int64_t>(s.b) * a.n_step + step) * a.q_stride +
                                                            static_cast<int64_t>(s.head * a.group + h) * D)[c];
                }
            }
#pragma unroll
            for (int u = 0; u < QV; ++u) {
                const int i = (WAYS == 1 ? threadIdx.x : tid) + u * Q_THREADS, r = i / (D / 8), c = i % (D / 8);
                uint4 q = q_v[u];
                if (FP8) {                       // f16 times a power of two a row; the D / 8 threads of a row are neighbours in a warp
                    const uint32_t x[4] = {q.x, q.y, q.z, q.w};
                    float f[8], top = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        f[e] = __uint_as_float(e & 1 ? x[e >> 1] & 0xFFFF0000u : x[e >> 1] << 16);
                        top = fmaxf(top, fabsf(f[e]));
                    }
#pragma unroll
                    for (int o = D / 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
                    const int exponent = min(max(static_cast<int>(__float_as_uint(top) >> 23), 1), 253);      // top in [2^(exponent - 127), 2 of that)
                    const float down = __uint_as_float(static_cast<uint32_t>(254 - exponent) << 23);
                    if (c == 0) st_shared_f32(row_s + (q_block * kWayRows + r) * 4, __uint_as_float(static_cast<uint32_t>(exponent) << 23));
                    q = make_uint4(pack_f16(f[0] * down, f[1] * down), pack_f16(f[2] * down, f[3] * down), pack_f16(f[4] * down, f[5] * down),
                                   pack_f16(f[6] * down, f[7] * down));
                }
                st_shared_v4(q_s + (q_block * (D / 64) + (c >> 3)) * (kWayRows * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4), q);
            }
            fence_proxy_async_smem();
            mbar_arrive(bar_q + 8 * q_block);
            if (FP8) threads_sync(WAYS == 1 ? 1 : 1 + w, Q_THREADS);

            const int row = row0 + tid % R, step = min(row / a.group, a.n_step - 1), key0 = tid / R * R;      // first key of the copy's (of a warp)
            const int sees = len - (a.n_step - 1 - step), sees_least = len - (a.n_step - 1 - row0 / a.group);
            const float row_scale = FP8 ? p.scale_log2 * ld_shared_f32(row_s + (q_block * kWayRows + tid) * 4) : p.scale_log2;
            constexpr int T0 = WAYS == 1 ? 1 : 0, STEP = WAYS == 1 ? 2 : 1;    // WAYS == 1: the ways take tiles in turn
            float m = -INFINITY, l = 0.f;
            for (int t = T0 * w; t < s.n; t += STEP) {
                const int vi = 2 * (it + t) + 1, v_slot = vi % NS;
                const uint32_t pos_at = pos_s + ((it + t) % kPosTiles) * 32;
                // Scores first: a way that had no rows in a segment before this one would take an older phase of the slot's barrier for its own. V's arrival
                // publishes the positions; the slot's next copy waits for this tile's probabilities.
                if (!wait(bar_s + 8 * w, n_s++ & 1) || !wait(bar_full + 8 * v_slot, (vi / NS) & 1)) break;
                tcgen05_fence_after_sync();
                int pos = 0;
                if (lane < per_tile) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(pos) : "r"(pos_at + lane * 4) : "memory");
                const bool clean = __all_sync(0xFFFFFFFFu, lane >= per_tile || (pos >= 0 && pos + piece <= sees_least));
                if (!FP8 && (WAYS == 1 || w == 0) && !clean) {
                    // rows of V that no token sees meet probability 0 and may hold anything: they are cleared, for way 1 too, whose product follows way 0's
                    const int first = __shfl_sync(0xFFFFFFFFu, pos, tid >> piece_log2);
                    if (first < 0 || first + (tid & (piece - 1)) >= len) {
#pragma unroll
                        for (int c = 0; c < D / 8; ++c)
                            st_shared_v4(slots + v_slot * L::kSlotBytes + (c >> 3) * L::kBlock + tid * 128 + ((c & 7) << 4), make_uint4(0u, 0u, 0u, 0u));
                        fence_proxy_async_smem();
                    }
                }
                const uint32_t sc_at = scale_s + ((it + t) % kScaleTiles) * (3 * kTile * 4) + key0 * 4;
                uint32_t x[NX][32];
#pragma unroll
                for (int c = 0; c < NX; ++c) tmem_ld_32x32b_x32(s_col + key0 + 32 * c, x[c]);
#pragma unroll
                for (int c = 0; c < NX; ++c) tmem_ld_wait(x[c]);
                if (FP8) {
#pragma unroll
                    for (int g = 0; g < R / 4; ++g) {                            // four keys
                        const float4 k_sc = ld_shared_f32x4(sc_at + g * 16);
                        uint32_t* y = &x[g / 8][g % 8 * 4];
                        y[0] = __float_as_uint(__uint_as_float(y[0]) * k_sc.x);
                        y[1] = __float_as_uint(__uint_as_float(y[1]) * k_sc.y);
                        y[2] = __float_as_uint(__uint_as_float(y[2]) * k_sc.z);
                        y[3] = __float_as_uint(__uint_as_float(y[3]) * k_sc.w);
                    }
                }
                float scale = row_scale;
                if (!clean || (!FP8 && !(scale > 0.f))) {
#pragma unroll
                    for (int g = 0; g < R / 16; ++g) {                        // 16 keys
                        const int k = key0 + g * 16, first = __shfl_sync(0xFFFFFFFFu, pos, k >> piece_log2);
                        const int n = first < 0 ? 0 : sees - first - (k & (piece - 1));
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            uint32_t& y = x[g / 2][g % 2 * 16 + e];
                            y = __float_as_uint(e < n ? __uint_as_float(y) * scale : -INFINITY);
                        }
                    }
                    scale = 1.f;
                }
                float top4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                if (FP8) {
#pragma unroll
                    for (int g = 0; g < R / 4; ++g) {
                        const float4 above = ld_shared_f32x4(sc_at + kTile * 4 + g * 16);
                        const uint32_t* y = &x[g / 8][g % 8 * 4];
                        top4[0] = fmaxf(top4[0], fmaf(__uint_as_float(y[0]), scale, above.x));
                        top4[1] = fmaxf(top4[1], fmaf(__uint_as_float(y[1]), scale, above.y));
                        top4[2] = fmaxf(top4[2], fmaf(__uint_as_float(y[2]), scale, above.z));
                        top4[3] = fmaxf(top4[3], fmaf(__uint_as_float(y[3]), scale, above.w));
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < NX; ++c)
#pragma unroll
                        for (int e = 0; e < 32; ++e) top4[e & 3] = fmaxf(top4[e & 3], __uint_as_float(x[c][e]));
                }
                float top = fmaxf(fmaxf(top4[0], top4[1]), fmaxf(top4[2], top4[3]));
                if (!FP8) top *= scale;
                if (__any_sync(0xFFFFFFFFu, !(top <= m + kSlack))) {
                    const float v = fmaxf(m, top), f = exp2_fast(m - (v == -INFINITY ? 0.f : v));
                    m = v;
                    l *= f;
                    if (t >= STEP) {                                          // the scores are there, so the way's products before them are done
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
                for (int c = 0; c < R / 16; ++c) {                            // 16 keys
                    uint32_t y[8];
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        float v[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            v[k] = exp2_fast(fmaf(__uint_as_float(x[c / 2][c % 2 * 16 + 2 * e + k]), scale, -use));
                            sum[k] += v[k];
                        }
                        if (FP8) {
                            const float4 v_sc = ld_shared_f32x4(sc_at + 2 * kTile * 4 + (c * 16 + 2 * e) * 4);
                            y[e] = pack_f16(v[0] * v_sc.x, v[1] * v_sc.y);
                            y[e + 1] = pack_f16(v[2] * v_sc.z, v[3] * v_sc.w);
                        } else {
                            y[e] = pack_bf16(v[0], v[1]);
                            y[e + 1] = pack_bf16(v[2], v[3]);
                        }
                    }
                    tmem_st_32x32b_x8(s_col + key0 / 2 + 8 * c, y);
                }
                if (COPIES > 1) {                                             // the other copies' keys
                    const uint32_t none[8] = {};
#pragma unroll
                    for (int c = 0; c < kTile / 16; ++c)
                        if (8 * c < key0 / 2 || 8 * c >= (key0 + R) / 2) tmem_st_32x32b_x8(s_col + 8 * c, none);
                }
                l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
                tmem_st_wait();
                tcgen05_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_p + 8 * w);
            }
            it += s.n;
            const bool any = WAYS == 2 || w < s.n;                            // (one tile: the second way has none)
            if (any) wait(bar_o + 8 * w, n_o++ & 1);
            tcgen05_fence_after_sync();
            // ---- output
            const bool writes = ok && row < rows_all;
            const int64_t out_row = (static_cast<int64_t>(s.b) * a.n_step + step) * a.H + s.head * a.group + (row - step * a.group);
            const int64_t piece_row = (static_cast<int64_t>(blockIdx.x) * 2 + (s.t0 == 0 ? 1 : 0)) * kBlockRows + q_block * kWayRows + tid % R;
            float over = 1.f;
            auto put = [&](int c, const uint32_t(&o)[32]) {                   // columns c .. c + 31 of the row
                if (!writes) return;
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
            };
            auto put_sums = [&]() {
                if (!writes) return;
                if (!whole) p.part_ml[piece_row] = make_float2(m, l);
                else if (a.lse) a.lse[out_row] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
            };
            if (WAYS == 2) {
                if (whole) over = l == 0.f ? 0.f : 1.f / (kHead * l);
                const uint32_t rows_at = q_s + w * (D / 64) * (kWayRows * 128);
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    uint32_t o[32];
                    tmem_ld_32x32b_x32(o_col + c, o);
                    tmem_ld_wait(o);
                    if (!whole) {
                        put(c, o);
                        continue;
                    }
                    // A row's 16-byte vectors go through the place of its q, so that neighbours write neighbouring ones.
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint32_t v[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) v[k] = pack_bf16(__uint_as_float(o[8 * e + 2 * k]) * over, __uint_as_float(o[8 * e + 2 * k + 1]) * over);
                        const int at = c / 8 + e;
                        st_shared_v4(rows_at + (at >> 3) * (kWayRows * 128) + tid * 128 + (((at & 7) ^ (tid & 7)) << 4), make_uint4(v[0], v[1], v[2], v[3]));
                    }
                }
                put_sums();
                if (whole) {
                    threads_sync(1 + w, 128);
                    for (int i = tid; i < kWayRows * (D / 8); i += 128) {
                        const int r = i / (D / 8), c = i % (D / 8);
                        if (!ok || row0 + r >= rows_all) break;
                        const int st = (row0 + r) / a.group;
                        const int64_t to = (static_cast<int64_t>(s.b) * a.n_step + st) * a.H + s.head * a.group + (row0 + r - st * a.group);
                        reinterpret_cast<uint4*>(a.out + to * D)[c] = ld_shared_v4(rows_at + (c >> 3) * (kWayRows * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4));
                    }
                    threads_sync(1 + w, 128);
                }
            } else {
                // All parts of a row, two ways' and the copies', go through shared memory, a quarter of the columns at a time, in place of q, which the
                // products are done with: [column][thread], so that neighbours meet in no bank.
                threads_sync(1, 256);
                st_shared_f32x2(q_s + threadIdx.x * 8, m, l);
                threads_sync(1, 256);
                const int r = threadIdx.x % R;
                float best = -INFINITY;
                l = 0.f;
#pragma unroll
                for (int part = 0; part < 2 * COPIES; ++part) best = fmaxf(best, ld_shared_f32x2(q_s + (part * R + r) * 8).x);
                const float use = best == -INFINITY ? 0.f : best, f = exp2_fast(m - use);
#pragma unroll
                for (int part = 0; part < 2 * COPIES; ++part) {
                    const float2 ml = ld_shared_f32x2(q_s + (part * R + r) * 8);
                    l = fmaf(ml.y, exp2_fast(ml.x - use), l);
                }
                m = best;
                if (whole) over = l == 0.f ? 0.f : 1.f / (kHead * l);
                threads_sync(1, 256);
                constexpr int CW = D / 4, CT = CW / (2 * COPIES);             // columns of a turn; of a thread that sums
                const int c0 = static_cast<int>(threadIdx.x) / R * CT;
#pragma unroll 1
                for (int c = 0; c < D; c += CW) {
                    if (any) {
                        uint32_t o[CW];
                        tmem_ld_columns(o_col + c, o);
                        tmem_ld_wait(o);
#pragma unroll
                        for (int e = 0; e < CW; ++e) st_shared_f32(q_s + (e * 256 + threadIdx.x) * 4, __uint_as_float(o[e]) * f);
                    } else {
#pragma unroll
                        for (int e = 0; e < CW; ++e) st_shared_f32(q_s + (e * 256 + threadIdx.x) * 4, 0.f);
                    }
                    threads_sync(1, 256);
                    float v[CT];
#pragma unroll
                    for (int e = 0; e < CT; ++e) {
                        v[e] = 0.f;
#pragma unroll
                        for (int part = 0; part < 2 * COPIES; ++part) v[e] += ld_shared_f32(q_s + ((c0 + e) * 256 + part * R + r) * 4);
                    }
                    if (writes) {
#pragma unroll
                        for (int e = 0; e < CT; e += 2) {
                            if (whole) *reinterpret_cast<uint32_t*>(a.out + out_row * D + c + c0 + e) = pack_bf16(v[e] * over, v[e + 1] * over);
                            else *reinterpret_cast<float2*>(p.part_o + piece_row * D + c + c0 + e) = make_float2(v[e], v[e + 1]);
                        }
                    }
                    threads_sync(1, 256);
                }
                if (threadIdx.x < R) put_sums();
            }
            tcgen05_fence_before_sync();         // (the next segment's first product follows this thread's next arrival)
        }
        if (!ok) give_up(DEV_TIMEOUT_EPILOGUE);
        if (threadIdx.x == 0) p.owners[blockIdx.x] = owner;
        // Blocks of rows that see no key: zeros and -inf.
        const int blocks = H_kv * p.row_blocks;
        for (int64_t u = blockIdx.x; u < static_cast<int64_t>(a.B) * blocks; u += gridDim.x) {
            const int b = static_cast<int>(u / blocks), of = static_cast<int>(u - static_cast<int64_t>(b) * blocks);
            const int head = of / p.row_blocks, r = of - head * p.row_blocks;
            if (tiles_of_block(p, b, r) != 0) continue;
            for (int i = threadIdx.x; i < kBlockRows * (D / 8); i += kSoftmaxWarps * 32) {
                const int row = r * kBlockRows + i / (D / 8);
                if (row >= rows_all) break;
                const int step = row / a.group;
                const int64_t to = (static_cast<int64_t>(b) * a.n_step + step) * a.H + head * a.group + (row - step * a.group);
                reinterpret_cast<uint4*>(a.out + to * D)[i % (D / 8)] = make_uint4(0u, 0u, 0u, 0u);
                if (a.lse && i % (D / 8) == 0) a.lse[to] = -INFINITY;
            }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(L::kOtherRegs));
        if (warp == kProducerWarp) {
            // ------------------------------------------------------------ producer: K and V of a tile into the next two places of the ring
            constexpr int ROWB = D * (FP8 ? 1 : 2), INNER = ROWB >= 128 ? 128 : ROWB;      // bytes of a cached row; of a row of one copy
            const uint32_t piece_bytes = static_cast<uint32_t>(piece) * (ROWB + (FP8 ? 4 : 0));
            const int P = a.c.page_size;
            int it = 0;                          // tiles
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
                        const unsigned v = static_cast<unsigned>(s.t0) * kTile + (static_cast<unsigned>(i) << piece_log2);
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
                    for (int t = 0; ok && t < n_here; ++t, ++it) {
                        const bool mine = (lane >> per_tile_log2) == t;
                        const int in_tile = lane & (per_tile - 1);
                        const uint32_t bytes = __popc(__ballot_sync(0xFFFFFFFFu, mine && now.pos >= 0)) * piece_bytes;
#pragma unroll
                        for (int kv = 0; kv < 2; ++kv) {
                            const int i = 2 * it + kv, at = i % NR;
                            if (i >= NR && !wait(bar_raw_empty + 8 * at, ((i / NR) & 1) ^ 1)) break;
                            if (kv == 0 && mine)
                                asm volatile("st.shared.b32 [%0], %1;" ::"r"(pos_s + (it % kPosTiles) * 32 + in_tile * 4), "r"(now.pos) : "memory");
                            __syncwarp();
                            const uint32_t full = bar_raw + 8 * at;
                            if (lane == 0) mbar_arrive_expect_tx(full, bytes);
                            __syncwarp();
                            if (mine && now.pos >= 0) {
                                const uint32_t to = raws + at * (FP8 ? L::kRawBytes : L::kSlotBytes) + in_tile * piece * INNER;
#pragma unroll
                                for (int h = 0; h < ROWB / INNER; ++h)
                                    tma_load_4d(to + h * L::kBlock, kv ? &v_map : &k_map, full, h * 64, now.off, s.head, now.page);
                                if (FP8)
                                    bulk_load_1d(raws + at * L::kRawBytes + L::kCodes + in_tile * piece * 4,
                                                 (kv ? a.c.v_scale : a.c.k_scale) + (static_cast<int64_t>(now.page) * H_kv + s.head) * P + now.off, piece * 4, full);
                            }
                        }
                    }
                }
            }
            if (!ok) give_up(DEV_TIMEOUT_PRODUCER);
        } else if (warp == kProductsWarp) {
            // ------------------------------------------------------------ products
            constexpr uint32_t kFormat = FP8 ? 0 : 1;
            constexpr uint32_t kIdescS = umma_idesc(kFormat, kFormat, 128, kTile), kIdescO = umma_idesc(kFormat, kFormat, 128, D) | kUmmaBMajorMN;
            uint32_t n_q[2] = {0u, 0u}, n_p[2] = {0u, 0u};
            int it = 0;
            auto wait_mma = [&](uint32_t bar, uint32_t parity) {
                const bool there = wait(bar, parity);
                tcgen05_fence_after_sync();
                return there;
            };
            auto scores = [&](int w, int i, bool last) {                      // place i of the ring; the last reader
                const int slot = i % NS;
                if (!wait_mma(bar_full + 8 * slot, (i / NS) & 1)) return;
#pragma unroll
                for (int h = 0; h < D / 64; ++h)
                    umma_f16_x4<2, 2>(tmem + 128 * w, umma_smem_desc_sw128(q_s + ((WAYS == 1 ? 0 : w) * (D / 64) + h) * kWayRows * 128),
                                      umma_smem_desc_sw128(slots + slot * L::kSlotBytes + h * L::kBlock), kIdescS, h > 0);
                umma_commit_elect(bar_s + 8 * w);
                if (last) umma_commit_elect(bar_empty + 8 * slot);
            };
            auto values = [&](int w, int i, bool first, bool last, bool end) {      // the way's first, its last
                const int slot = i % NS;
                if (!wait_mma(bar_p + 8 * w, n_p[w]++ & 1) || !wait_mma(bar_full + 8 * slot, (i / NS) & 1)) return;
                const uint64_t v_desc = umma_smem_desc_sw128_mn(slots + slot * L::kSlotBytes, L::kBlock);
#pragma unroll
                for (int k = 0; k < kTile / 16; ++k)
                    umma_f16_ts_elect_acc(tmem + L::kColO + D * w, tmem + 128 * w + 8 * k, v_desc + k * 128, kIdescO, !first || k > 0);
                if (last) umma_commit_elect(bar_empty + 8 * slot);
                if (end) umma_commit_elect(bar_o + 8 * w);
            };
            Walk walk(p, run);
            Segment s;
            while (ok && walk.next(s)) {
                const int i0 = 2 * it;
                if (WAYS == 1) {
                    wait_mma(bar_q, n_q[0]++ & 1);
                    for (int t = 0; ok && t < s.n + 2; ++t) {
                        const int w = t & 1;
                        if (t >= 2 && t - 2 < s.n) {
                            if (w == 0) values(0, i0 + 2 * t - 3, t < 4, true, t >= s.n);
                            else values(1, i0 + 2 * t - 3, t < 4, true, t >= s.n);
                        }
                        if (ok && t < s.n) scores(w, i0 + 2 * t, true);
                    }
                } else {
                    const int ways = ways_of(s);
                    for (int t = 0; ok && t <= s.n; ++t) {
#pragma unroll
                        for (int w = 0; w < 2; ++w) {
                            if (w >= ways) break;
                            if (t > 0) values(w, i0 + 2 * t - 1, t == 1, w == ways - 1, t == s.n);
                            if (t == 0) wait_mma(bar_q + 8 * w, n_q[w]++ & 1);
                            if (ok && t < s.n) scores(w, i0 + 2 * t, w == ways - 1);
                        }
                    }
                }
                it += s.n;
            }
            if (!ok) give_up(DEV_TIMEOUT_MMA);
        } else if (FP8 && warp < kConvertWarp + kConvertWarps) {
            // ------------------------------------------------------------ codes to f16 (exact), scales to what the softmax takes
            const int tid = threadIdx.x - kConvertWarp * 32;
            constexpr int CH = D / 16;           // 16-byte chunks of codes of a row
            int it = 0;
            Walk walk(p, run);
            Segment s;
            while (ok && walk.next(s)) {
                const int len = length_of(a, s.b);
                for (int i = 2 * it; i < 2 * (it + s.n); ++i) {
                    const int at = i % NR, slot = i % NS, tile = i >> 1;
                    const bool is_v = i & 1;
                    if (!wait(bar_raw + 8 * at, (i / NR) & 1)) break;
                    if (i >= NS && !wait(bar_empty + 8 * slot, ((i / NS) & 1) ^ 1)) break;
                    int pos = 0;
                    if (lane < per_tile) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(pos) : "r"(pos_s + (tile % kPosTiles) * 32 + lane * 4) : "memory");
                    // rows of V that no token sees meet probability 0 and may hold anything: they become zeros, their scales 1
                    const bool clean = !is_v || __all_sync(0xFFFFFFFFu, lane >= per_tile || (pos >= 0 && pos + piece <= len));
                    auto unseen = [&](int r) {
                        const int first = __shfl_sync(0xFFFFFFFFu, pos, r >> piece_log2);
                        return first < 0 || first + (r & (piece - 1)) >= len;
                    };
                    const uint32_t from = raws + at * L::kRawBytes, to = slots + slot * L::kSlotBytes;
                    // Four chunks at a time: row and chunk of the first, the others follow 512 / CH rows on.
                    const int r0 = tid / CH, c = tid % CH;
                    // A row's chunks c and c + 4 of d = 128 would meet in the same banks: the second four write their halves the other way round.
                    const int turn = c >> 2, c2 = 2 * (c & 3);
                    const uint32_t block = to + turn * L::kBlock;
#pragma unroll 1
                    for (int u0 = 0; u0 < CH; u0 += 4) {
                        uint4 x[4];
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            const int r = r0 + (u0 + u) * (128 / CH);
                            x[u] = ld_shared_v4(from + (D == 128 ? r * 128 + ((c ^ (r & 7)) << 4) : r * 64 + ((c ^ ((r >> 1) & 3)) << 4)));
                        }
                        if (!clean) {
#pragma unroll
                            for (int u = 0; u < 4; ++u)
                                if (unseen(r0 + (u0 + u) * (128 / CH))) x[u] = make_uint4(0u, 0u, 0u, 0u);
                        }
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            const int r = r0 + (u0 + u) * (128 / CH);
                            uint4 lo, hi;
                            lo.x = e4m3x2_to_f16x2(x[u].x & 0xFFFFu);
                            lo.y = e4m3x2_to_f16x2(x[u].x >> 16);
                            lo.z = e4m3x2_to_f16x2(x[u].y & 0xFFFFu);
                            lo.w = e4m3x2_to_f16x2(x[u].y >> 16);
                            hi.x = e4m3x2_to_f16x2(x[u].z & 0xFFFFu);
                            hi.y = e4m3x2_to_f16x2(x[u].z >> 16);
                            hi.z = e4m3x2_to_f16x2(x[u].w & 0xFFFFu);
                            hi.w = e4m3x2_to_f16x2(x[u].w >> 16);
                            st_shared_v4(block + r * 128 + (((c2 + turn) ^ (r & 7)) << 4), turn ? hi : lo);
                            st_shared_v4(block + r * 128 + (((c2 + 1 - turn) ^ (r & 7)) << 4), turn ? lo : hi);
                        }
                    }
                    float sc = ld_shared_f32(from + L::kCodes + tid * 4);
                    if (!clean && unseen(tid)) sc = 1.f;
                    const uint32_t sc_to = scale_s + (tile % kScaleTiles) * (3 * kTile * 4) + tid * 4;
                    if (is_v) {
                        st_shared_f32(sc_to + kTile * 4, log2_above(sc));
                        st_shared_f32(sc_to + 2 * kTile * 4, sc * kF16Head);
                    } else {
                        st_shared_f32(sc_to, sc);
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(bar_full + 8 * slot);
                        mbar_arrive(bar_raw_empty + 8 * at);
                    }
                }
                it += s.n;
            }
            if (!ok) give_up(DEV_TIMEOUT_GATHER);
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
    if (warp == kProductsWarp) {
        tcgen05_fence_after_sync();
        tmem_dealloc(tmem, 512);
    }
}

template <int D, bool FP8, int WAYS, int R>
cudaError_t run_rows(const CUtensorMap& k_map, const CUtensorMap& v_map, const Params& p, int grid, cudaStream_t stream, int* launches) {
    using L = Layout<D, FP8, WAYS>;
    const auto kernel = paged_rows_kernel<D, FP8, WAYS, R>;
    cudaError_t e = ensure_max_dynamic_smem(reinterpret_cast<const void*>(kernel), L::kBytes);
    if (e != cudaSuccess) return e;
    *launches += 1;
    e = launch_behind(kernel, dim3(grid), L::kThreads, L::kBytes, stream, k_map, v_map, p);
    if (e != cudaSuccess) return e;
    constexpr int kBlockRows = WAYS == 1 ? R : 2 * kWayRows;
    const int all = p.a.n_step * p.a.group, rows = all < kBlockRows ? all : kBlockRows;
    *launches += 1;
    const float out_scale = FP8 ? 1.f / kF16Head : 1.f;
    if (grid > 12 * static_cast<int64_t>(p.a.B) * p.a.c.H_kv * p.row_blocks)      // many pieces a unit, as in paged_attn.cu
        return launch_behind(paged_merge_kernel<D, kBlockRows, 4, 2>, dim3(grid, (rows + 1) / 2), 256, 0, stream, p, out_scale);
    return launch_behind(paged_merge_kernel<D, kBlockRows, 1, 4>, dim3(grid, (rows + 3) / 4), 128, 0, stream, p, out_scale);
}

}  // namespace

cudaError_t launch_paged_attn_rows(const PagedAttnArgs& a, void* workspace, const CUtensorMap& k_map, const CUtensorMap& v_map, unsigned int* status,
                                   int sm_count, cudaStream_t stream, int* launches) {
    Params p{};
    p.a = a;
    p.ways = a.n_step * a.group > kWayRows ? 2 : 1;
    const int rows = a.n_step * a.group, block = rows <= 64 ? 64 : p.ways * kWayRows;
    p.row_blocks = (rows + block - 1) / block;
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
#define IDXC_RUN(D_, F_)                                                                    \
    (block == 64    ? run_rows<D_, F_, 1, 64>(k_map, v_map, p, grid, stream, launches)       \
     : block == 128 ? run_rows<D_, F_, 1, 128>(k_map, v_map, p, grid, stream, launches)      \
                    : run_rows<D_, F_, 2, 128>(k_map, v_map, p, grid, stream, launches))
    if (a.c.d == 128) return a.c.fp8 ? IDXC_RUN(128, true) : IDXC_RUN(128, false);
    return a.c.fp8 ? IDXC_RUN(64, true) : IDXC_RUN(64, false);
#undef IDXC_RUN
}

}  // namespace idxc
