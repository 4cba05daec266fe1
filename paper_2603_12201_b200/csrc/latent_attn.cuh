// What the kernels of the attention over latent rows share: their arguments, and a group's walk over its run of tiles.
#pragma once

#include <cuda_bf16.h>

#include "kernels.h"
#include "latent_format.cuh"
#include "ptx_sm100.cuh"

namespace idxc {
namespace latent {

constexpr int kTile = 64;                           // cache rows of a tile (2^6)
constexpr int kRows = 64;                           // query rows of a CTA
constexpr int kBlocks = 9;                          // 64-column blocks of a row
// A loader of Q waits while the piece before is worked on: its bound grows with that piece (a tile takes a few thousand cycles).
__device__ __forceinline__ long long piece_budget(int tiles) { return kWaitCycleBudget + 50000LL * tiles; }
// First cache row of sequence b.
__device__ __forceinline__ int64_t first_row(const LatentArgs& a, int64_t b) { return a.kv_base ? near_base(__ldg(a.kv_base + b), a.n_kv) : 0; }
constexpr float kMoveThreshold = 8.f;               // log2 units: probabilities stay below 2^8 of the reference

// Tiles of a unit: counted beforehand, or from its sequence's length (no lengths: max_len for all). A unit of a prompt chunk walks all tiles of its
// sequence, those behind its last token's position too: their scores are masked away. (Units that stop there had half the tiles of a whole prompt and were no
// faster, 1061 -> 1088 us for 2048 tokens: equal runs of tiles then give short units to the first groups, and each costs a piece's end.)
struct UnitTiles {
    const int32_t* counted;      // [units] or nullptr
    const int32_t* lens;
    int64_t max_len;
    uint32_t blocks_per_seq;     // units of a sequence
    int tile_log2;               // rows of a tile
    __device__ __forceinline__ uint32_t seq_of(uint32_t unit) const { return blocks_per_seq == 1 ? unit : unit / blocks_per_seq; }
    __device__ __forceinline__ int operator()(uint32_t unit) const {
        if (counted) return *static_cast<const volatile int32_t*>(counted + unit);      // (not __ldg: written while this kernel may already run)
        const int most = static_cast<int>(max_len), len = lens ? __ldg(lens + seq_of(unit)) : most;      // (max_len <= 2^30)
        return (min(max(len, 0), most) + (1 << tile_log2) - 1) >> tile_log2;
    }
};

struct Params {
    LatentArgs a;
    UnitTiles tiles;
    int2* starts;                // [groups] (unit, tile) at which a group's run begins
    int32_t* runs;               // [groups + 1] first tile of the run in the end-to-end order (both written by the kernel for the merge)
    uint32_t units;              // (sequence, block of 64 * ways query rows)
    int blocks_per_seq;          // units of a sequence
    int ways;                    // CTAs of a group: 1 or 2, each 64 rows
    int groups;
    float scale_log2;            // |scale| * log2(e), 1 for a zero scale
    float sign;                  // 1, -1 or 0: scores are multiplied by it first
    __nv_bfloat16* out;
    float* lse;
    float* part_out;             // [groups][2][ways][64][512]
    float* part_lse;             // [groups][2][ways][64]
    unsigned int* status;
};

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// ---------------------------------------------------------------- the run of a group, and its walk over it
// The tiles of all units, laid end to end, are cut into `groups` runs, as a rule of equal length (to within one). Every CTA finds its own by a
// scan over the units, which costs about a microsecond where a kernel of its own before this one costs five.
// Up to 128 units every warp does that by itself, four units a lane, without a barrier: their loads (early_tiles) are under way while the
// CTA sets itself up.
constexpr uint32_t kFewUnits = 128;
struct EarlyTiles { int n[4]; };
__device__ __forceinline__ EarlyTiles early_tiles(uint32_t units, const UnitTiles& tiles) {
    const uint32_t first = 4 * (threadIdx.x & 31);
    EarlyTiles e;
#pragma unroll
    for (int k = 0; k < 4; ++k) e.n[k] = units <= kFewUnits && first + k < units ? tiles(first + k) : 0;
    return e;
}
// Brings the first 4 KB of kv_base to the L1 (every role loads its sequence's when it starts).
__device__ __forceinline__ void early_bases(const int64_t* kv_base, int64_t B) {
    const int64_t at = 16 * static_cast<int64_t>(threadIdx.x & 31);
    if (kv_base != nullptr && at < B)
        asm volatile("{\n\t.reg .b64 x;\n\tld.global.nc.b64 x, [%0];\n\t}" ::"l"(kv_base + at));
}
struct Run {
    uint32_t unit;        // where it begins
    int t;
    int first, n, total;  // first tile end to end, number of tiles, tiles of all units
};
__device__ __forceinline__ void cut_run(Run& r, int group, int groups) {
    const int each = r.total / groups, more = r.total - each * groups;       // total * group / groups without 64-bit divisions
    r.first = each * group + more * group / groups;
    r.n = each * (group + 1) + more * (group + 1) / groups - r.first;
}
// `cut_tiles`: what a run that begins or ends inside a unit costs more than one that does not, in tiles (its output goes out in fp32
// and through the merge). Few units that are alike are therefore not cut evenly: with s = groups / units >= 1 each unit is cut by itself into s
// runs, with s = 0 a run takes whole units, where the longest such run is no longer than an even one and that.
__device__ __forceinline__ Run find_run(uint32_t units, const UnitTiles& tiles, const EarlyTiles& early, int group, int groups, int cut_tiles,
                                        int* scratch /* shared, 40 words */) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
    if (units <= kFewUnits) {
        const int sum = (early.n[0] + early.n[1]) + (early.n[2] + early.n[3]);
        const int longest = __reduce_max_sync(0xFFFFFFFFu, max(max(early.n[0], early.n[1]), max(early.n[2], early.n[3])));
        int incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xFFFFFFFFu, incl, o);
            if (lane >= o) incl += y;
        }
        Run r{0, 0, 0, 0, 0};
        r.total = __shfl_sync(0xFFFFFFFFu, incl, 31);
        // first tile of unit u, end to end, and its tiles
        auto unit_at = [&](int u, int& n) -> int {
            const int k = u & 3;
            const int mine = incl - sum + (k > 0 ? early.n[0] : 0) + (k > 1 ? early.n[1] : 0) + (k > 2 ? early.n[2] : 0);
            n = __shfl_sync(0xFFFFFFFFu, k == 0 ? early.n[0] : (k == 1 ? early.n[1] : (k == 2 ? early.n[2] : early.n[3])), (u >> 2) & 31);
            return u < 4 * 32 ? __shfl_sync(0xFFFFFFFFu, mine, (u >> 2) & 31) : r.total;
        };
        const int n_units = static_cast<int>(units), s = groups / n_units;
        const long long apart = s > 0 ? (longest + s - 1) / s : static_cast<long long>((n_units + groups - 1) / groups) * longest;
        if (apart <= r.total / groups + cut_tiles) {
            int n, n_end;
            if (s > 0) {
                const int u = group / s, p = group - u * s;
                const int at = unit_at(min(u, n_units - 1), n);
                const int t0 = static_cast<int>(static_cast<uint32_t>(n) * p / s), t1 = static_cast<int>(static_cast<uint32_t>(n) * (p + 1) / s);
                const bool idle = u >= n_units;
                r.unit = idle ? 0 : static_cast<uint32_t>(u);
                r.t = idle ? 0 : t0;
                r.first = idle ? r.total : at + t0;
                r.n = idle ? 0 : t1 - t0;
            } else {
                const int u0 = group * n_units / groups, u1 = (group + 1) * n_units / groups;
                r.unit = static_cast<uint32_t>(u0);
                r.first = unit_at(u0, n);
                r.n = unit_at(u1, n_end) - r.first;
            }
            return r;
        }
        cut_run(r, group, groups);
        int before = incl - sum, unit = -1, t = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (r.first >= before && r.first < before + early.n[k]) {
                unit = 4 * lane + k;
                t = r.first - before;
            }
            before += early.n[k];
        }
        const uint32_t who = __ballot_sync(0xFFFFFFFFu, unit >= 0);
        if (who != 0) {
            r.unit = static_cast<uint32_t>(__shfl_sync(0xFFFFFFFFu, unit, __ffs(who) - 1));
            r.t = __shfl_sync(0xFFFFFFFFu, t, __ffs(who) - 1);
        }
        return r;
    }
    const uint32_t n_thr = blockDim.x;
    int mine = 0;                                    // this thread's unit of the first block of units
    int sum = 0;
    for (uint32_t u = threadIdx.x; u < units; u += n_thr) {
        const int n = tiles(u);
        if (u < n_thr) mine = n;
        sum += n;
    }
    sum = __reduce_add_sync(0xFFFFFFFFu, sum);
    if (lane == 0) scratch[warp] = sum;
    __syncthreads();
    Run r{0, 0, 0, 0, 0};
    for (int w = 0; w < n_warps; ++w) r.total += scratch[w];
    cut_run(r, group, groups);
    if (r.n > 0) {                                   // (uniform over the CTA)
        int before_block = 0;
        for (uint32_t u0 = 0; u0 < units; u0 += n_thr) {
            const uint32_t u = u0 + threadIdx.x;
            const int n = u0 == 0 ? mine : (u < units ? tiles(u) : 0);
            int incl = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xFFFFFFFFu, incl, o);
                if (lane >= o) incl += y;
            }
            __syncthreads();                         // (the last readers of scratch are done)
            if (lane == 31) scratch[warp] = incl;
            __syncthreads();
            int before = before_block + incl - n, all = 0;
            for (int w = 0; w < n_warps; ++w) {
                if (w < warp) before += scratch[w];
                all += scratch[w];
            }
            if (r.first >= before && r.first < before + n) {
                scratch[32] = static_cast<int>(u);
                scratch[33] = r.first - before;
            }
            before_block += all;
            if (r.first < before_block) break;
        }
        __syncthreads();
        r.unit = static_cast<uint32_t>(scratch[32]);
        r.t = scratch[33];
    }
    __syncthreads();
    return r;
}

struct Piece {
    uint32_t unit;
    int t0, n;            // first tile, number of tiles
    bool whole;           // all tiles of the unit
};
struct Walk {
    const UnitTiles& tiles;
    uint32_t unit;
    int t, left;
    __device__ __forceinline__ Walk(const UnitTiles& tl, const Run& r) : tiles(tl), unit(r.unit), t(r.t), left(r.n) {}
    __device__ __forceinline__ bool next(Piece& pc) {
        if (left <= 0) return false;
        int nt = tiles(unit);
        while (nt == 0) nt = tiles(++unit);                 // left > 0: a unit with tiles follows
        pc.unit = unit;
        pc.t0 = t;
        pc.n = min(nt - t, left);
        pc.whole = t == 0 && pc.n == nt;
        left -= pc.n;
        ++unit;
        t = 0;
        return true;
    }
};

// A warp's 32 rows of 16 N bytes, a row in each lane's registers, to global memory through 512 N bytes of shared memory: an
// instruction then writes 32 / N rows in contiguous pieces. (Stored straight from the registers, 16 bytes of 32 rows an instruction, the
// output of a piece took 10 to 12 thousand clocks.) dst(r, i): where piece i of row r goes, nullptr: nowhere.
template <int N, typename Dst>
__device__ __forceinline__ void store_rows(uint32_t stage, int lane, const uint4 (&v)[N], Dst dst) {
    auto swizzle = [](int r) -> int { return N == 8 ? (r & 7) : ((r >> 1) & 3); };
#pragma unroll
    for (int i = 0; i < N; ++i) st_shared_v4(stage + lane * (16 * N) + ((i ^ swizzle(lane)) << 4), v[i]);
    __syncwarp();
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int r = k * (32 / N) + lane / N, i = lane % N;
        const uint4 w = ld_shared_v4(stage + r * (16 * N) + ((i ^ swizzle(r)) << 4));
        uint4* to = dst(r, i);
        if (to != nullptr) *to = w;
    }
    __syncwarp();
}

// Zeros and -inf for the units without tiles; every group looks at its share, a lane each. `quarter`: which of the four calling warps.
template <typename RowsOf>
__device__ __forceinline__ void write_empty_units(const Params& p, int group, int quarter, int lane, int seq_rows, RowsOf rows_of) {
    for (int64_t u0 = group; u0 < p.units; u0 += 32 * static_cast<int64_t>(p.groups)) {
        const int64_t mine = u0 + lane * static_cast<int64_t>(p.groups);
        uint32_t none = __ballot_sync(0xFFFFFFFFu, mine < p.units && p.tiles(static_cast<uint32_t>(mine < p.units ? mine : 0)) == 0);
        for (; none; none &= none - 1) {
            int64_t seq;
            int r0;
            const int n = rows_of(static_cast<uint32_t>(u0 + (__ffs(none) - 1) * static_cast<int64_t>(p.groups)), seq, r0);
            for (int r = quarter; r < n; r += 4) {
                const int64_t at = seq * seq_rows + r0 + r;
                reinterpret_cast<uint4*>(p.out + at * 512)[lane] = make_uint4(0, 0, 0, 0);
                reinterpret_cast<uint4*>(p.out + at * 512)[32 + lane] = make_uint4(0, 0, 0, 0);
                if (p.lse && lane == 0) p.lse[at] = -INFINITY;
            }
        }
    }
}

}  // namespace latent

// latent_attn_pair.cu: units of more than 64 query rows, a CTA pair each (maps: see LatentMaps).
cudaError_t launch_latent_attn_pair(const LatentMaps& maps, const latent::Params& p, cudaStream_t stream);

}  // namespace idxc
