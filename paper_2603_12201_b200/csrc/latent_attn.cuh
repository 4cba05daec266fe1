// What the kernels of the attention over latent rows share: their arguments, and a group's walk over its run of tiles.
#pragma once

#include <cuda_bf16.h>

#include "kernels.h"
#include "latent_format.cuh"
#include "ptx_sm100.cuh"

namespace idxc {
namespace latent {

constexpr int kTile = 64;                           // cache rows of a tile
constexpr int kRows = 64;                           // query rows of a CTA
constexpr int kBlocks = 9;                          // 64-column blocks of a row
constexpr float kMoveThreshold = 8.f;               // log2 units: probabilities stay below 2^8 of the reference

struct Params {
    LatentArgs a;
    const int32_t* tiles;        // [units] tiles of every unit
    const int2* starts;          // [groups + 1] (unit, tile) at which a group's run begins
    const int32_t* runs;         // [groups + 1] first tile of the run in the end-to-end order
    int64_t units;               // (sequence, block of 64 * ways query rows)
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

// ---------------------------------------------------------------- the walk of a group over its run
struct Piece {
    int64_t unit;
    int t0, n;            // first tile, number of tiles
    bool whole;           // all tiles of the unit
};
struct Walk {
    const int32_t* tiles;
    int64_t unit;
    int t, left;
    __device__ __forceinline__ Walk(const Params& p, int group) : tiles(p.tiles), unit(0), t(0), left(__ldg(p.runs + group + 1) - __ldg(p.runs + group)) {
        if (left > 0) {
            const int2 s = __ldg(p.starts + group);
            unit = s.x;
            t = s.y;
        }
    }
    __device__ __forceinline__ bool next(Piece& pc) {
        if (left <= 0) return false;
        int nt = __ldg(tiles + unit);
        while (nt == 0) nt = __ldg(tiles + ++unit);         // left > 0: a unit with tiles follows
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

// Zeros and -inf for the units without tiles; every group looks at its share, a lane each. `quarter`: which of the four calling warps.
template <typename RowsOf>
__device__ __forceinline__ void write_empty_units(const Params& p, int group, int quarter, int lane, int seq_rows, RowsOf rows_of) {
    for (int64_t u0 = group; u0 < p.units; u0 += 32 * static_cast<int64_t>(p.groups)) {
        const int64_t mine = u0 + lane * static_cast<int64_t>(p.groups);
        uint32_t none = __ballot_sync(0xFFFFFFFFu, mine < p.units && __ldg(p.tiles + (mine < p.units ? mine : 0)) == 0);
        for (; none; none &= none - 1) {
            int64_t seq;
            int r0;
            const int n = rows_of(u0 + (__ffs(none) - 1) * static_cast<int64_t>(p.groups), seq, r0);
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
