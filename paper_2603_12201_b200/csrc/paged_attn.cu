// Attention of new tokens over their requests' pages of keys and values, H / H_kv query heads to a key head:
//     x[s] = scale <q, k_s> over the visible keys s,   out = sum_s softmax(x)[s] v_s,   lse = log sum_s exp(x[s])
// over all pages of a request, or over the pages that a selection names for each (request, key head).
//
// What bounds it: a key and a value of d columns are 4 d bytes (bf16) and 4 d flops a query row; with the 1 to 32 rows that share a key head
// in a decode step that is 1 to 32 flops a byte, far below the tensor cores' 200: HBM. So the design serves the copies. One CTA an SM, a ring of
// 64-key tiles of K and V (32 KB in bf16 with d = 128) filled by TMA from whole pages or 16-key pieces of them, and warp-level MMAs, which take
// their operands from shared memory with one ldmatrix each and keep scores, softmax and output in registers: 128 MMAs a tile and 16 rows, of which
// the tensor cores issue several times what the copies deliver. (A tile is the M = 16 rows of up to 16 query rows; tcgen05's M = 64 or 128 would
// be mostly padding, and its accumulators would cross tensor memory twice a tile.)
//
// Each of 8 warps takes 16 or 32 keys of a tile and up to 32 query rows (with more rows, 2 or 4 warps the same keys) with its own running
// maximum and sum; the warps meet once at a segment's end. The tiles of all (request, key head, block of rows), end to end, are cut into equal runs, a run a
// CTA, which finds it from the lengths on the device; segments cut by a run's end go to the workspace in fp32 and through a merge kernel. All sums
// have an order fixed by the sizes, so results repeat bit for bit.
//
// e4m3 rows: codes become f16 (exact) on the way to the registers, with q as f16 times a power of two a row (its largest element in [1, 2); what
// falls below f16's range is below 2^-25 of that, an fp32 rounding). The value's scale goes into the probability, whose reference is the running
// maximum of x + log2(scale), rounded up: probability times scale then stays in f16's range however the scales differ.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "kernels.h"
#include "ptx_sm100.cuh"

namespace idxc {
namespace {

constexpr int kTile = 64;                       // keys of a tile
constexpr int kProducerRegs = 40;
constexpr float kF16Head = 16384.f;             // probabilities times scale reach 1; f16 holds them times 2^14

struct Params {
    PagedAttnArgs a;
    int row_blocks;              // blocks of MAXR query rows of a (request, key head)
    int piece_log2;              // keys of a copy: 16, 32 or 64
    float scale_log2;            // scale * log2(e)
    float* part_o;               // [grid][2][MAXR][D]
    float2* part_ml;             // [grid][2][MAXR] (maximum in log2 units, sum)
    int4* owners;                // [grid] the segment that begins in a CTA's run and does not end in it: (request, unit, its tiles in the run, all), request -1: none
    int* total;                  // tiles of the call
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
__device__ __forceinline__ void st_shared_f32x2(uint32_t addr, float x, float y) {
    asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(addr), "f"(x), "f"(y) : "memory");
}
__device__ __forceinline__ void st_shared_v2(uint32_t addr, uint32_t x, uint32_t y) {
    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(addr), "r"(x), "r"(y) : "memory");
}
// log2 of a positive scale, rounded up, as a number between -60 and 60.
__device__ __forceinline__ float log2_above(float scale) {
    return static_cast<float>(min(max(static_cast<int>(__float_as_uint(scale) >> 23 & 255u) - 126, -60), 60));
}
template <int WARPS>
__device__ __forceinline__ void consumers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(WARPS * 32) : "memory"); }

// ---------------------------------------------------------------- work
// Keys of request b that the call knows of.
__device__ __forceinline__ int length_of(const PagedAttnArgs& a, int b) { return min(max(__ldg(a.lens + b), 0), static_cast<int>(a.max_len)); }
// Tiles of one (key head, block of rows) of request b: of its keys, or of the first min(n_sel, pages of the request) entries of its selection.
__device__ __forceinline__ int tiles_of(const PagedAttnArgs& a, int b) {
    const int len = length_of(a, b);
    if (!a.pages) return (len + kTile - 1) / kTile;
    const int pages = (len + a.c.page_size - 1) / a.c.page_size;
    return static_cast<int>((static_cast<int64_t>(min(a.n_sel, pages)) * a.c.page_size + kTile - 1) / kTile);
}
struct Run {
    int b, x;             // request, tile among all of the request's units
    int n;                // tiles
    int total;
};
// First tile of a CTA's run: total * cta / n, cut among n = min(grid, total) CTAs so that no run in front of another is empty.
__device__ __forceinline__ int run_begin(int total, int cta, int grid) {
    const int n = min(grid, total);
    if (cta >= n) return total;
    const unsigned each = static_cast<unsigned>(total) / n, more = total - each * n;
    return static_cast<int>(each * cta + more * cta / n);
}
__device__ __forceinline__ Run find_run(const Params& p, int* scratch /* shared, 16 words */) {
    const int units = p.a.c.H_kv * p.row_blocks;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_thr = blockDim.x, n_warps = n_thr >> 5;
    int sum = 0, mine = 0;
    for (int b = threadIdx.x; b < p.a.B; b += n_thr) {
        const int n = tiles_of(p.a, b) * units;
        if (b < n_thr) mine = n;
        sum += n;
    }
    sum = __reduce_add_sync(0xFFFFFFFFu, sum);
    if (lane == 0) scratch[warp] = sum;
    __syncthreads();
    Run r{0, 0, 0, 0};
    for (int w = 0; w < n_warps; ++w) r.total += scratch[w];
    const int first = run_begin(r.total, blockIdx.x, gridDim.x);
    r.n = run_begin(r.total, blockIdx.x + 1, gridDim.x) - first;
    if (r.n > 0) {                               // (uniform over the CTA)
        int before_block = 0;
        for (int b0 = 0; b0 < p.a.B; b0 += n_thr) {
            const int b = b0 + threadIdx.x;
            const int n = b0 == 0 ? mine : (b < p.a.B ? tiles_of(p.a, b) * units : 0);
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
                scratch[12] = b;
                scratch[13] = first - before;
            }
            before_block += all;
            if (first < before_block) break;
        }
        __syncthreads();
        r.b = scratch[12];
        r.x = scratch[13];
    }
    return r;
}
struct Segment {
    int b, unit;          // request; key head * row_blocks + block of rows
    int t0, n, nt;        // first tile, tiles here, tiles of the unit
};
struct Walk {
    const Params& p;
    int b, x, left, nt;
    __device__ __forceinline__ Walk(const Params& q, const Run& r) : p(q), b(r.b), x(r.x), left(r.n), nt(r.n > 0 ? tiles_of(q.a, r.b) : 0) {}
    __device__ __forceinline__ bool next(Segment& s) {
        if (left <= 0) return false;
        const int units = p.a.c.H_kv * p.row_blocks;
        while (x == nt * units) {                // the request's end (or one without tiles); more tiles follow
            nt = tiles_of(p.a, ++b);
            x = 0;
        }
        s.b = b;
        s.unit = x / nt;
        s.t0 = x - s.unit * nt;
        s.n = min(nt - s.t0, left);
        s.nt = nt;
        x += s.n;
        left -= s.n;
        return true;
    }
};

// ---------------------------------------------------------------- shared memory
// Up to 32 query rows: 4 consumer warps a CTA and two CTAs an SM, so that one's segment end hides behind the other's tiles. More rows: 8 and
// one. A fifth (ninth) warp is the producer; three more fill up its warpgroup, because registers are handed out by warpgroups: the launch's
// 128 (168) a thread, of which the producer's keeps 40.
template <int D, bool FP8, int MT, int RG>
struct Layout {
    static constexpr int kWarps = RG == 1 ? 4 : 8;
    static constexpr int kThreads = (kWarps + 4) * 32;
    static constexpr int kCtas = RG == 1 ? 2 : 1;                      // of an SM
    static constexpr int kConsumerRegs = RG == 1 ? 216 : 232;
    static_assert(128 * kProducerRegs + kWarps * 32 * kConsumerRegs <= kThreads * (RG == 1 ? 128 : 168), "shares of the launch's registers");
    static constexpr int kRows = 16 * MT * RG;                         // query rows of a CTA
    static constexpr int kParts = kWarps / RG;                         // warps that share a row
    static constexpr int kKeys = D == 128 && !FP8 && RG < 4 ? 16 : 32; // keys of a tile that a warp takes
    static constexpr int kSplit = kTile / kKeys;                       // warps (of a row) that share a tile
    static constexpr int kSlots = kParts / kSplit;                     // tiles worked on at a time
    static constexpr int kTileBytes = kTile * D * (FP8 ? 1 : 2);
    static constexpr int kStageBytes = 2 * kTileBytes + (FP8 ? 1024 : 0);      // K, V, scales of K and of V (256 bytes each)
    static constexpr int kSlice = MT == 1 ? 32 : 16;                   // columns of the output that go through shared memory at a time
    static constexpr int kPitch = kSlice + 8;                          // floats between rows there: no bank conflicts on float2
    static constexpr int kQBytes = kRows * D * 2;
    static constexpr int kRedBytes = kWarps * MT * 16 * kPitch * 4;
    static constexpr int kShared = kQBytes > kRedBytes ? kQBytes : kRedBytes;  // q, and the output's slices when q is done with
    static constexpr int kMlBytes = kWarps * MT * 16 * 8;
    static constexpr int kSmall = 1024 + 1536;                         // alignment of the stages; barriers, positions, scales of q
    static constexpr int kLimit = (233472 - kCtas * (1024 + 128)) / kCtas;     // an SM's, without what the system and static arrays take
    static constexpr int kFit = (kLimit - kSmall - kShared - kMlBytes) / kStageBytes;
    // A stage belongs to one slot, whose warps see every phase of its barrier: were the stages no multiple of the slots, a warp could come to
    // a stage's barrier while the tile before its own is still on the way, and take the parity of the one before that for its own.
    static constexpr int kStages = (kFit > 24 ? 24 : kFit) / kSlots * kSlots;
    static constexpr int kBytes = kSmall + kStages * kStageBytes + kShared + kMlBytes;
    static_assert(kParts >= kSplit, "the warps of a row take a whole tile");
    static_assert(kStages >= 3 && kStages % kSlots == 0, "a ring of at least three tiles, each stage one slot's");
    static_assert(kStages * (16 + 16) + kRows * 4 + 16 <= 1536, "small words");
};

// Byte offset of 16-byte chunk `c` of row `r` in a tile whose rows are at most 128 bytes (wider ones lie in blocks of 128).
template <int ROW_BYTES>
__device__ __forceinline__ uint32_t chunk_at(int r, int c) {
    if (ROW_BYTES >= 128) return (c >> 3) * (kTile * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4);
    return r * 64 + ((c ^ ((r >> 1) & 3)) << 4);
}

template <int D, bool FP8, int MT, int RG>
__global__ void __launch_bounds__((Layout<D, FP8, MT, RG>::kThreads), (Layout<D, FP8, MT, RG>::kCtas))
paged_attn_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const __grid_constant__ Params p) {
    using L = Layout<D, FP8, MT, RG>;
    constexpr int ROWB = D * (FP8 ? 1 : 2);      // bytes of a cached row
    constexpr int NS = L::kStages, W = L::kWarps;
    extern __shared__ uint8_t raw[];
    const uint32_t base = smem_u32(raw);
    const uint32_t stages = (base + 1023u) & ~1023u;
    const uint32_t q_s = stages + NS * L::kStageBytes;
    const uint32_t red_s = q_s;
    const uint32_t ml_s = q_s + L::kShared;
    const uint32_t bars = ml_s + L::kMlBytes;    // full[NS], empty[NS]
    const uint32_t pos_s = bars + NS * 16;       // [NS][4] position of the first key of each piece, -1: none
    const uint32_t qs_s = pos_s + NS * 16;       // [kRows] power of two taken out of a row of q
    const uint32_t flag_s = qs_s + L::kRows * 4;
    __shared__ int scratch[16];
    volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(raw + (flag_s - base));

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < NS; ++s) {
            mbar_init(bars + 8 * s, 1);
            mbar_init(bars + 8 * (NS + s), RG * L::kSplit);
        }
        *abort_flag = 0;
        fence_mbar_init();
        tma_prefetch_desc(&k_map);
        tma_prefetch_desc(&v_map);
    }
    let_next_start();
    wait_for_previous();
    const Run run = find_run(p, scratch);        // (its barriers publish the mbarriers too)
    const PagedAttnArgs& a = p.a;
    if (threadIdx.x == 0 && blockIdx.x == 0) *p.total = run.total;

    if (warp >= W) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kProducerRegs));
        if (warp > W) return;
        // ------------------------------------------------------------ producer: pieces of pages into the ring
        const int piece = 1 << p.piece_log2, per_tile_log2 = 6 - p.piece_log2, per_tile = 1 << per_tile_log2;
        const uint32_t piece_bytes = static_cast<uint32_t>(piece) * (2 * ROWB + (FP8 ? 8 : 0));
        const int P = a.c.page_size;
        int it = 0;
        Walk walk(p, run);
        Segment s;
        while (walk.next(s)) {
            const int len = length_of(a, s.b);
            const int head = s.unit / p.row_blocks;
            const int32_t* table = a.table + static_cast<int64_t>(s.b) * a.ld_table;
            const int32_t* sel = a.pages ? a.pages + (static_cast<int64_t>(s.b) * a.c.H_kv + head) * a.n_sel : nullptr;
            const int n_entries = (len + P - 1) / P;      // pages of the request; with a selection min(n_sel, that) entries are looked at
            const int most = sel ? min(a.n_sel, n_entries) : n_entries;
            const int n_pieces = s.n << per_tile_log2;
            struct Where { int page, off, pos; };
            auto locate = [&](int i) -> Where {           // piece i of the segment
                Where w{0, 0, -1};
                if (i < n_pieces) {
                    const unsigned v = static_cast<unsigned>(s.t0) * kTile + (static_cast<unsigned>(i) << p.piece_log2);
                    const unsigned e = v / static_cast<unsigned>(P);
                    w.off = static_cast<int>(v - e * P);
                    if (static_cast<int>(e) < most) {
                        const int logical = sel ? __ldg(sel + e) : static_cast<int>(e);
                        if (logical >= 0 && logical < n_entries) {
                            const int pos = logical * P + w.off;
                            w.page = __ldg(table + logical);
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
                    if (mine) asm volatile("st.shared.b32 [%0], %1;" ::"r"(pos_s + st * 16 + in_tile * 4), "r"(now.pos) : "memory");
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
                            tma_load_4d(k_to + h * (kTile * INNER) + at, &k_map, full, h * 64, now.off, head, now.page);
                            tma_load_4d(v_to + h * (kTile * INNER) + at, &v_map, full, h * 64, now.off, head, now.page);
                        }
                        if (FP8) {
                            const int64_t from = (static_cast<int64_t>(now.page) * a.c.H_kv + head) * P + now.off;
                            const uint32_t sc = v_to + L::kTileBytes + in_tile * piece * 4;
                            bulk_load_1d(sc, a.c.k_scale + from, piece * 4, full);
                            bulk_load_1d(sc + 256, a.c.v_scale + from, piece * 4, full);
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
        return;
    }

    // ---------------------------------------------------------------- consumers
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(L::kConsumerRegs));
    const int rg = warp % RG, part = warp / RG;
    const int slot = part / L::kSplit, key0 = (part % L::kSplit) * L::kKeys;      // this warp's keys of its slot's tiles
    const int g = lane >> 2, j = lane & 3;       // row and column pair of the fragments
    const int rows_all = a.n_step * a.group;
    constexpr int KS = L::kKeys;
    constexpr int NT = D / 8;                    // output fragments of 8 columns
    int it = 0;
    bool ok = true;
    Walk walk(p, run);
    Segment s;
    int4 owner = make_int4(-1, 0, 0, 0);
    while (walk.next(s)) {
        const int len = length_of(a, s.b);
        const int head = s.unit / p.row_blocks, row0 = (s.unit - head * p.row_blocks) * L::kRows;
        const int n_rows = min(rows_all - row0, L::kRows);
        const bool whole = s.t0 == 0 && s.n == s.nt;
        // q of the segment, zeros behind the last row
        for (int i = threadIdx.x; i < L::kRows * (D / 8); i += W * 32) {
            const int r = i / (D / 8), c = i - r * (D / 8);
            uint4 x = make_uint4(0u, 0u, 0u, 0u);
            if (r < n_rows) {
                const int step = (row0 + r) / a.group, h = row0 + r - step * a.group;
                x = __ldg(reinterpret_cast<const uint4*>(a.q + (static_cast<int64_t>(s.b) * a.n_step + step) * a.q_stride +
                                                         static_cast<int64_t>(head * a.group + h) * D) + c);
            }
            const uint32_t row_at = q_s + r * (D * 2);
            if (!FP8) {
                st_shared_v4(row_at + ((c ^ (r & 7)) << 4), x);
            } else {
                // the D / 8 threads of a row are neighbours in a warp
                const uint32_t* w = &x.x;
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
                if (c == 0) asm volatile("st.shared.f32 [%0], %1;" ::"r"(qs_s + r * 4), "f"(__uint_as_float(static_cast<uint32_t>(exponent) << 23)) : "memory");
                uint32_t h[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) h[e] = pack_f16(f[2 * e] * down, f[2 * e + 1] * down);
                // Of 16 columns lane j of a fragment takes 4 j .. 4 j + 3 (the four codes of a register of K): pairs 0 and 1 of each four
                // go to places 2 j and 2 j + 8.
                const int block = c >> 1, odd = c & 1;                 // 16 columns; the second eight of them
                const uint32_t lo = row_at + (((2 * block) ^ (r & 7)) << 4) + odd * 8, hi = row_at + (((2 * block + 1) ^ (r & 7)) << 4) + odd * 8;
                st_shared_v2(lo, h[0], h[2]);
                st_shared_v2(hi, h[1], h[3]);
            }
        }
        consumers_sync<W>();

        // Address of this lane's row for an A fragment of q: matrices (rows 0-7, 8-15) x (columns 0-7, 8-15).
        auto q_frag = [&](int mt, int ks, uint32_t(&f)[4]) {
            const int r = (rg * MT + mt) * 16 + (lane & 15), c = 2 * ks + (lane >> 4);
            ldmatrix_x4(q_s + r * (D * 2) + ((c ^ (r & 7)) << 4), f);
        };
        uint32_t qf[MT == 1 ? D / 16 : 1][4];
        if (MT == 1) {
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) q_frag(0, ks, qf[MT == 1 ? ks : 0]);
        }
        int sees[MT][2];                         // keys that the row of fragment half h sees
        float row_scale[MT][2];
        float m[MT][2], l[MT][2];
        float o[MT][NT][4];
        int sees_least = len;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = (rg * MT + mt) * 16 + h * 8 + g;
                sees[mt][h] = len - (a.n_step - 1 - min((row0 + r) / a.group, a.n_step - 1));
                row_scale[mt][h] = FP8 ? p.scale_log2 * ld_shared_f32(qs_s + r * 4) : p.scale_log2;
                m[mt][h] = -INFINITY;
                l[mt][h] = 0.f;
            }
        sees_least = len - (a.n_step - 1);       // (of the request's first token)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[mt][n][e] = 0.f;

        // first tile of the segment whose place in the run is this warp's
        for (int t = (slot - it % L::kSlots + L::kSlots) % L::kSlots; t < s.n; t += L::kSlots) {
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
            int at[KS / 16];                     // position of the first key of each 16
            int last = 0;
#pragma unroll
            for (int i = 0; i < KS / 16; ++i) {
                const int key = key0 + i * 16, pc = key >> p.piece_log2;
                int first;
                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(first) : "r"(pos_s + st * 16 + pc * 4) : "memory");
                at[i] = first < 0 ? INT32_MAX / 2 : first + (key - (pc << p.piece_log2));
                last = max(last, at[i] + 16);
            }
            const bool clean = last <= sees_least;
            if (!clean) {
                // Rows of V that no token sees meet probability 0 and may hold anything: they are cleared.
                const int r = key0 + (lane & (KS - 1)), i = (lane & (KS - 1)) >> 4;
                const int first = KS == 16 || i == 0 ? at[0] : at[KS / 16 - 1];
                if (first + (r & 15) >= len) {
#pragma unroll
                    for (int c = lane / KS; c < ROWB / 16; c += 32 / KS) st_shared_v4(v_at + chunk_at<ROWB>(r, c), make_uint4(0u, 0u, 0u, 0u));
                    if (FP8) asm volatile("st.shared.f32 [%0], %1;" ::"r"(sc_at + 256 + r * 4), "f"(1.f) : "memory");
                    fence_proxy_async_smem();    // (the next copy into these rows comes from the asynchronous proxy)
                }
                __syncwarp();
            }
            {
                float x[MT][KS / 8][4];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int n = 0; n < KS / 8; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[mt][n][e] = 0.f;
                // scores: an ldmatrix takes 8 keys x 64 bytes
                constexpr int STEPS = FP8 ? 4 : 2;        // 16-column steps in 64 bytes
#pragma unroll
                for (int c4 = 0; c4 < ROWB / 64; ++c4) {
                    uint32_t qa[STEPS][MT][4];
#pragma unroll
                    for (int u = 0; u < STEPS; ++u)
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            if (MT == 1) {
#pragma unroll
                                for (int e = 0; e < 4; ++e) qa[u][mt][e] = qf[MT == 1 ? c4 * STEPS + u : 0][e];
                            } else {
                                q_frag(mt, c4 * STEPS + u, qa[u][mt]);
                            }
                        }
#pragma unroll
                    for (int n = 0; n < KS / 8; ++n) {
                        uint32_t kb[4];
                        ldmatrix_x4(k_at + chunk_at<ROWB>(key0 + n * 8 + (lane & 7), c4 * 4 + (lane >> 3)), kb);
#pragma unroll
                        for (int u = 0; u < STEPS; ++u) {
                            uint32_t b0, b1;
                            if (FP8) {
                                b0 = e4m3x2_to_f16x2(kb[u] & 0xFFFFu);
                                b1 = e4m3x2_to_f16x2(kb[u] >> 16);
                            } else {
                                b0 = kb[(2 * u) & 3];
                                b1 = kb[(2 * u + 1) & 3];
                            }
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt) mma_16816<FP8>(x[mt][n], qa[u][mt], b0, b1);
                        }
                    }
                }
                // softmax: x becomes probabilities (times the value's scale for 8 bits)
                float vs[FP8 ? KS / 8 : 1][2];
#pragma unroll
                for (int n = 0; n < KS / 8; ++n) {
                    float2 k_sc = make_float2(1.f, 1.f);
                    if (FP8) {
                        k_sc = ld_shared_f32x2(sc_at + (key0 + n * 8 + 2 * j) * 4);
                        const float2 v2 = ld_shared_f32x2(sc_at + 256 + (key0 + n * 8 + 2 * j) * 4);
                        vs[FP8 ? n : 0][0] = v2.x;
                        vs[FP8 ? n : 0][1] = v2.y;
                    }
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            float v = x[mt][n][e] * row_scale[mt][e >> 1];
                            if (FP8) v *= e & 1 ? k_sc.y : k_sc.x;
                            if (!clean && at[n >> 1] + ((n & 1) * 8 + 2 * j + (e & 1)) >= sees[mt][e >> 1]) v = -INFINITY;
                            x[mt][n][e] = v;
                        }
                }
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    float top[2] = {m[mt][0], m[mt][1]};
#pragma unroll
                    for (int n = 0; n < KS / 8; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) top[e >> 1] = fmaxf(top[e >> 1], FP8 ? x[mt][n][e] + log2_above(vs[FP8 ? n : 0][e & 1]) : x[mt][n][e]);
                    float use[2];
                    bool moved = false;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        top[h] = fmaxf(top[h], __shfl_xor_sync(0xFFFFFFFFu, top[h], 1));
                        top[h] = fmaxf(top[h], __shfl_xor_sync(0xFFFFFFFFu, top[h], 2));
                        use[h] = top[h] == -INFINITY ? 0.f : top[h];
                        moved |= top[h] != m[mt][h];
                    }
                    if (__any_sync(0xFFFFFFFFu, moved)) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const float f = exp2_fast(m[mt][h] - use[h]);
                            l[mt][h] *= f;
                            m[mt][h] = top[h];
#pragma unroll
                            for (int n = 0; n < NT; ++n) {
                                o[mt][n][2 * h] *= f;
                                o[mt][n][2 * h + 1] *= f;
                            }
                        }
                    }
#pragma unroll
                    for (int n = 0; n < KS / 8; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float pr = exp2_fast(x[mt][n][e] - use[e >> 1]);
                            l[mt][e >> 1] += pr;
                            x[mt][n][e] = FP8 ? pr * (vs[FP8 ? n : 0][e & 1] * kF16Head) : pr;
                        }
                }
                // output
#pragma unroll
                for (int kk = 0; kk < KS / 16; ++kk) {
                    uint32_t pa[MT][4];
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float lo = x[mt][2 * kk + (e >> 1)][2 * (e & 1)], hi = x[mt][2 * kk + (e >> 1)][2 * (e & 1) + 1];
                            pa[mt][e] = FP8 ? pack_f16(lo, hi) : pack_bf16(lo, hi);
                        }
                    const int r = key0 + kk * 16 + (lane & 15);      // matrices (keys 0-7, 8-15) x two 16-byte chunks
#pragma unroll
                    for (int c2 = 0; c2 < ROWB / 32; ++c2) {
                        uint32_t vb[4];
                        ldmatrix_x4_trans(v_at + chunk_at<ROWB>(r, 2 * c2 + (lane >> 4)), vb);
                        if (!FP8) {
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt) {
                                mma_16816<false>(o[mt][(2 * c2) % NT], pa[mt], vb[0], vb[1]);
                                mma_16816<false>(o[mt][(2 * c2 + 1) % NT], pa[mt], vb[2], vb[3]);
                            }
                        } else {
                            // A register holds columns 2 g, 2 g + 1 of keys 2 j, 2 j + 1: the even column's pair of keys, then the odd one's.
#pragma unroll
                            for (int u = 0; u < 2; ++u) {
                                const uint32_t w0 = __byte_perm(vb[2 * u], 0, 0x3120), w1 = __byte_perm(vb[2 * u + 1], 0, 0x3120);
                                const uint32_t e0 = e4m3x2_to_f16x2(w0 & 0xFFFFu), e1 = e4m3x2_to_f16x2(w1 & 0xFFFFu);
                                const uint32_t d0 = e4m3x2_to_f16x2(w0 >> 16), d1 = e4m3x2_to_f16x2(w1 >> 16);
#pragma unroll
                                for (int mt = 0; mt < MT; ++mt) {
                                    mma_16816<true>(o[mt][(4 * c2 + 2 * u) % NT], pa[mt], e0, e1);
                                    mma_16816<true>(o[mt][(4 * c2 + 2 * u + 1) % NT], pa[mt], d0, d1);
                                }
                            }
                        }
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bars + 8 * (NS + st));
        }
        it += s.n;

        // ------------------------------------------------------------ the warps' parts of the segment joined
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                l[mt][h] += __shfl_xor_sync(0xFFFFFFFFu, l[mt][h], 1);
                l[mt][h] += __shfl_xor_sync(0xFFFFFFFFu, l[mt][h], 2);
                if (j == 0) st_shared_f32x2(ml_s + ((part * RG + rg) * MT * 16 + mt * 16 + h * 8 + g) * 8, m[mt][h], l[mt][h]);
            }
        consumers_sync<W>();
        const int64_t out_part = (static_cast<int64_t>(blockIdx.x) * 2 + (s.t0 == 0 ? 1 : 0)) * L::kRows;
        auto joined = [&](int r, float& top, float& sum) {          // r: row of the CTA
            const int of = r / (16 * MT), in = r % (16 * MT);
            top = -INFINITY;
            sum = 0.f;
            float2 v[L::kParts];
#pragma unroll
            for (int w = 0; w < L::kParts; ++w) {
                v[w] = ld_shared_f32x2(ml_s + ((w * RG + of) * MT * 16 + in) * 8);
                top = fmaxf(top, v[w].x);
            }
            const float use = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int w = 0; w < L::kParts; ++w) sum += v[w].y * exp2_fast(v[w].x - use);
        };
        float f[MT][2];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float top, sum;
                joined((rg * MT + mt) * 16 + h * 8 + g, top, sum);
                f[mt][h] = exp2_fast(m[mt][h] - (top == -INFINITY ? 0.f : top));
            }
        for (int r = threadIdx.x; r < n_rows; r += W * 32) {
            float top, sum;
            joined(r, top, sum);
            const float over = sum == 0.f ? 0.f : (FP8 ? 1.f / kF16Head : 1.f) / sum;
            asm volatile("st.shared.f32 [%0], %1;" ::"r"(qs_s + r * 4), "f"(over) : "memory");      // (q's scales are in registers)
            if (!whole) {
                p.part_ml[out_part + r] = make_float2(top, sum);
            } else if (a.lse) {
                const int step = (row0 + r) / a.group, h = row0 + r - step * a.group;
                a.lse[(static_cast<int64_t>(s.b) * a.n_step + step) * a.H + head * a.group + h] =
                    sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
            }
        }
#pragma unroll
        for (int c0 = 0; c0 < D; c0 += L::kSlice) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int n0 = 0; n0 < L::kSlice / 8; ++n0)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float v[2] = {o[mt][c0 / 8 + n0][2 * h] * f[mt][h], o[mt][c0 / 8 + n0][2 * h + 1] * f[mt][h]};
                        const uint32_t row = red_s + ((part * RG + rg) * MT * 16 + mt * 16 + h * 8 + g) * (L::kPitch * 4);
                        if (!FP8) {
                            st_shared_f32x2(row + (n0 * 8 + 2 * j) * 4, v[0], v[1]);
                        } else {                 // fragment 2 c + odd holds columns 16 c + 2 n + odd
                            const uint32_t to = row + ((n0 >> 1) * 16 + 4 * j + (n0 & 1)) * 4;
                            asm volatile("st.shared.f32 [%0], %1;" ::"r"(to), "f"(v[0]) : "memory");
                            asm volatile("st.shared.f32 [%0], %1;" ::"r"(to + 8), "f"(v[1]) : "memory");
                        }
                    }
            consumers_sync<W>();
            for (int i = threadIdx.x; i < n_rows * (L::kSlice / 2); i += W * 32) {
                const int r = i / (L::kSlice / 2), c = i % (L::kSlice / 2) * 2, of = r / (16 * MT), in = r % (16 * MT);
                float2 v = make_float2(0.f, 0.f);
#pragma unroll
                for (int w = 0; w < L::kParts; ++w) {
                    const float2 y = ld_shared_f32x2(red_s + ((w * RG + of) * MT * 16 + in) * (L::kPitch * 4) + c * 4);
                    v.x += y.x;
                    v.y += y.y;
                }
                if (!whole) {
                    *reinterpret_cast<float2*>(p.part_o + (out_part + r) * D + c0 + c) = v;
                } else {
                    const float over = ld_shared_f32(qs_s + r * 4);
                    const int step = (row0 + r) / a.group, h = row0 + r - step * a.group;
                    const int64_t to = ((static_cast<int64_t>(s.b) * a.n_step + step) * a.H + head * a.group + h) * D + c0 + c;
                    *reinterpret_cast<uint32_t*>(a.out + to) = pack_bf16(v.x * over, v.y * over);
                }
            }
            consumers_sync<W>();
        }
        if (s.t0 == 0 && !whole) owner = make_int4(s.b, s.unit, s.n, s.nt);
    }
    if (threadIdx.x == 0) p.owners[blockIdx.x] = owner;

    // Requests without keys: zeros and -inf.
    for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
        if (tiles_of(a, b) != 0) continue;
        const int64_t n_vec = static_cast<int64_t>(a.n_step) * a.H * (D / 8);
        uint4* to = reinterpret_cast<uint4*>(a.out + static_cast<int64_t>(b) * a.n_step * a.H * D);
        for (int64_t i = threadIdx.x; i < n_vec; i += W * 32) to[i] = make_uint4(0u, 0u, 0u, 0u);
        if (a.lse)
            for (int i = threadIdx.x; i < a.n_step * a.H; i += W * 32) a.lse[static_cast<int64_t>(b) * a.n_step * a.H + i] = -INFINITY;
    }
}

// Joins the pieces of a segment that runs cut. blockIdx.x: the CTA in whose run the segment begins; a warp a row.
template <int D, int ROWS>
__global__ void __launch_bounds__(128)
paged_merge_kernel(const __grid_constant__ Params p, int grid, float out_scale) {
    let_next_start();
    wait_for_previous();
    const int cta = blockIdx.x;
    const int4 own = p.owners[cta];
    if (own.x < 0) return;
    const int lane = threadIdx.x & 31, r = blockIdx.y * 4 + (threadIdx.x >> 5);
    const int head = own.y / p.row_blocks, row0 = (own.y - head * p.row_blocks) * ROWS;
    const int n_rows = min(p.a.n_step * p.a.group - row0, ROWS);
    if (r >= n_rows) return;
    const int total = *p.total;
    int pieces;                                  // the segment's tiles after this run fill the runs that follow
    {
        const int n = min(grid, total);
        const int last_tile = run_begin(total, cta + 1, grid) + (own.w - own.z) - 1;                    // end to end; in the run of
        const int last = static_cast<int>(((static_cast<int64_t>(last_tile) + 1) * n + total - 1) / total) - 1;      // the last c with total * c / n <= last_tile
        pieces = last - cta + 1;
    }
    auto row_of = [&](int i) -> int64_t { return (static_cast<int64_t>(cta + i) * 2 + (i == 0 ? 1 : 0)) * ROWS + r; };
    float top = -INFINITY;
    for (int i = lane; i < pieces; i += 32) top = fmaxf(top, p.part_ml[row_of(i)].x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    const float use = top == -INFINITY ? 0.f : top;
    constexpr int V = D / 32;                    // columns of a lane
    float acc[V] = {}, sum = 0.f;
    for (int i0 = 0; i0 < pieces; i0 += 32) {
        float w = 0.f, lw = 0.f;
        if (i0 + lane < pieces) {
            const float2 ml = p.part_ml[row_of(i0 + lane)];
            w = exp2_fast(ml.x - use);
            lw = w * ml.y;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) lw += __shfl_xor_sync(0xFFFFFFFFu, lw, o);
        sum += lw;
        const int n = min(32, pieces - i0);
#pragma unroll 4
        for (int i = 0; i < n; ++i) {
            const float wi = __shfl_sync(0xFFFFFFFFu, w, i);
            const float* from = p.part_o + row_of(i0 + i) * D + lane * V;
            if (V == 4) {
                const float4 y = *reinterpret_cast<const float4*>(from);
                acc[0] += wi * y.x;
                acc[1] += wi * y.y;
                acc[2 % V] += wi * y.z;
                acc[3 % V] += wi * y.w;
            } else {
                const float2 y = *reinterpret_cast<const float2*>(from);
                acc[0] += wi * y.x;
                acc[1] += wi * y.y;
            }
        }
    }
    const float over = sum == 0.f ? 0.f : out_scale / sum;
    const int step = (row0 + r) / p.a.group, h = row0 + r - step * p.a.group;
    const int64_t row = (static_cast<int64_t>(own.x) * p.a.n_step + step) * p.a.H + head * p.a.group + h;
    __nv_bfloat16* to = p.a.out + row * D + lane * V;
    if (V == 4) *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16(acc[0] * over, acc[1] * over), pack_bf16(acc[2 % V] * over, acc[3 % V] * over));
    else *reinterpret_cast<uint32_t*>(to) = pack_bf16(acc[0] * over, acc[1] * over);
    if (p.a.lse && lane == 0) p.a.lse[row] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
}

int max_grid(int cta_rows) { return cta_rows <= 32 ? 2 * kPagedMaxSms : kPagedMaxSms; }
int rows_of_cta(int rows) { return rows <= 16 ? 16 : (rows <= 32 ? 32 : (rows <= 64 ? 64 : 128)); }

template <int D, bool FP8, int MT, int RG>
cudaError_t run(const CUtensorMap& k_map, const CUtensorMap& v_map, Params& p, int sm_count, cudaStream_t stream, int* launches) {
    using L = Layout<D, FP8, MT, RG>;
    const int grid = sm_count * L::kCtas < max_grid(L::kRows) ? sm_count * L::kCtas : max_grid(L::kRows);
    auto kernel = paged_attn_kernel<D, FP8, MT, RG>;
    cudaError_t e = ensure_max_dynamic_smem(reinterpret_cast<const void*>(kernel), L::kBytes);
    if (e != cudaSuccess) return e;
    e = launch_behind(kernel, dim3(grid), L::kThreads, L::kBytes, stream, k_map, v_map, p);
    *launches += 1;
    if (e != cudaSuccess) return e;
    const int rows = p.a.n_step * p.a.group < L::kRows ? p.a.n_step * p.a.group : L::kRows;
    *launches += 1;
    return launch_behind(paged_merge_kernel<D, L::kRows>, dim3(grid, (rows + 3) / 4), 128, 0, stream, p, grid, FP8 ? 1.f / kF16Head : 1.f);
}

}  // namespace

// owners and total, the pieces' maxima and sums, the pieces
size_t paged_attn_workspace_bytes(int n_step, int group, int d) {
    const size_t rows = static_cast<size_t>(rows_of_cta(n_step * group)), grid = static_cast<size_t>(max_grid(static_cast<int>(rows)));
    return grid * 16 + 256 + grid * 2 * rows * (8 + static_cast<size_t>(d) * 4);
}
bool paged_attn_fits(const PagedAttnArgs& a) {
    const int64_t rows = static_cast<int64_t>(a.n_step) * a.group, cta = rows_of_cta(a.n_step * a.group);
    int64_t keys = a.max_len + kTile;
    if (a.pages) {
        const int64_t pages = (a.max_len + a.c.page_size - 1) / a.c.page_size;
        keys = (pages < a.n_sel ? pages : a.n_sel) * a.c.page_size + kTile;
    }
    return static_cast<double>(a.B) * a.c.H_kv * ((rows + cta - 1) / cta) * (keys / kTile) < 2147483648.0;
}

cudaError_t launch_paged_attn(const PagedAttnArgs& a, void* workspace, const CUtensorMap& k_map, const CUtensorMap& v_map, unsigned int* status,
                              int sm_count, cudaStream_t stream, int* launches) {
    Params p;
    p.a = a;
    const int rows = a.n_step * a.group, cta_rows = rows_of_cta(rows);
    p.row_blocks = (rows + cta_rows - 1) / cta_rows;
    p.piece_log2 = a.c.page_size % 64 == 0 ? 6 : (a.c.page_size % 32 == 0 ? 5 : 4);
    p.scale_log2 = a.scale * 1.4426950408889634f;
    uint8_t* w = static_cast<uint8_t*>(workspace);
    p.owners = reinterpret_cast<int4*>(w);
    const size_t grid = static_cast<size_t>(max_grid(cta_rows));
    p.total = reinterpret_cast<int*>(w + grid * 16);
    p.part_ml = reinterpret_cast<float2*>(w + grid * 16 + 256);
    p.part_o = reinterpret_cast<float*>(w + grid * 16 + 256 + grid * 2 * cta_rows * 8);
    p.status = status;
#define IDXC_RUN(D_, F_)                                                                                   \
    (cta_rows == 16   ? run<D_, F_, 1, 1>(k_map, v_map, p, sm_count, stream, launches)                          \
     : cta_rows == 32 ? run<D_, F_, 2, 1>(k_map, v_map, p, sm_count, stream, launches)                          \
     : cta_rows == 64 ? run<D_, F_, 2, 2>(k_map, v_map, p, sm_count, stream, launches)                          \
                      : run<D_, F_, 2, 4>(k_map, v_map, p, sm_count, stream, launches))
    if (a.c.d == 128) return a.c.fp8 ? IDXC_RUN(128, true) : IDXC_RUN(128, false);
    return a.c.fp8 ? IDXC_RUN(64, true) : IDXC_RUN(64, false);
#undef IDXC_RUN
}

}  // namespace idxc
