// Which cached positions of a sequence stay when its cache is cut to a budget: the newest `recent` ones, and among the older
// ones the budget - recent with the largest accumulated attention weight (ties: lowest position), in ascending order.
// A cluster of eight CTAs (or one, see the launch) takes a sequence, each an eighth of its positions, whose keys stay in shared memory (up to 48K positions a
// CTA; longer slices are read from global memory again). Three histogram passes (11 + 11 + 10 bits of an order-preserving key) find the
// key of the last position that stays exactly. The CTAs' counts are added up through distributed shared memory by one warp each, 64 bins at
// a time first and then the bins of one such group: 3 KB a pass, where all bins of all CTAs took 5000 clocks. Then every
// position's place in the output is the number of positions before it that stay, by prefix sums over lanes, warps and CTAs: no
// atomics on the output, ascending order for free. Bound by latency (five cluster barriers, and sweeps of a few microseconds that are
// instructions, not bytes): 8 sequences of 131072 positions 16 us, 24 of 6007 7 us (replayed back to back; 19 and 12 with cold caches).
#include "kernels.h"
#include "ptx_sm100.cuh"

namespace idxc {
namespace {

constexpr int kEvThreads = 1024;
constexpr int kEvWarps = kEvThreads / 32;
constexpr int kEvCtas = 8;                           // CTAs of a sequence, or one: see one_cta_each
constexpr int kEvBins = 2 * kEvThreads;               // 2048, two a thread
constexpr int kEvKeys = 49152;                       // keys of a slice that fit into shared memory at most
constexpr uint32_t kEvHistBytes = 2 * kEvBins * 4;

// Larger float = larger key; -0 and +0 share a key.
__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint2 ld_cluster_v2(uint32_t addr) {
    uint2 v;
    asm volatile("ld.shared::cluster.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
    return v;
}

// sum of n over the lanes up to this one
__device__ __forceinline__ uint32_t warp_scan(uint32_t n, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xFFFFFFFFu, n, o);
        if (lane >= o) n += y;
    }
    return n;
}

template <int CTAS>
__global__ void __launch_bounds__(kEvThreads)
evict_select_kernel(const float* acc, int64_t ld, const int32_t* lens, int budget, int recent, int key_slots,
                    int32_t* keep, int32_t* new_lens) {
    extern __shared__ __align__(16) uint32_t ev_smem[];
    uint32_t* hist = ev_smem;                        // [2][kEvBins]: this CTA's counts of a pass
    uint32_t* keys = hist + 2 * kEvBins;             // [key_slots]
    __shared__ __align__(8) uint32_t coarse[2][32];  // the same, 64 bins each
    __shared__ uint2 warp_count[kEvWarps];
    __shared__ uint32_t s_bin, s_left;
    __shared__ __align__(8) uint2 cta_count;         // positions of this CTA that certainly stay, and those at the border key
    wait_for_previous();
    let_next_start();
    auto sync_all = [&]() {                          // the CTAs of the sequence
        if (CTAS > 1) cluster_sync();
        else __syncthreads();
    };
    const int rank = CTAS > 1 ? static_cast<int>(cluster_ctarank()) : 0;
    const int b = blockIdx.x / CTAS, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int len = static_cast<int>(min(static_cast<int64_t>(max(lens[b], 0)), ld));
    const float* row = acc + b * ld;
    int32_t* out = keep + static_cast<int64_t>(b) * budget;
    const int stay = min(len, budget);
    if (tid == 0 && rank == 0) new_lens[b] = stay;
    for (int64_t j = stay + static_cast<int64_t>(rank) * kEvThreads + tid; j < budget; j += CTAS * kEvThreads) out[j] = -1;
    if (len <= budget) {                             // (the whole cluster leaves here together)
        for (int j = rank * kEvThreads + tid; j < len; j += CTAS * kEvThreads) out[j] = j;
        return;
    }
    const int old = len - recent;                    // positions that compete
    const int slice = ((len + CTAS - 1) / CTAS + 127) & ~127;
    const int p0 = min(rank * slice, len), p1 = min(p0 + slice, len);
    // a warp has a run of its CTA's slice, four positions a lane at a time
    const int seg = (((slice + kEvWarps - 1) / kEvWarps) + 127) & ~127;
    const int w0 = min(p0 + warp * seg, p1), w1 = min(w0 + seg, p1), w1_old = min(w1, old);
    // the key of a position that does not compete is 0, the lowest: it is never counted among those above another
    auto key_of = [&](int i) -> uint32_t { return i < w1_old ? order_key(row[i]) : 0u; };
    const bool kept = slice <= key_slots;
    if (kept) {
        for (int i = w0 + lane; i - lane < w1; i += 256) {        // eight loads under way at a time
            uint32_t k[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) k[e] = key_of(i + 32 * e);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (i - lane + 32 * (e & ~3) < w1) keys[i - p0 + 32 * e] = k[e];
        }
        __syncwarp();
    }
    // f(position of the first, four keys), the warp in step. (Rolled: with the keys in registers and the sweeps unrolled, every sweep waited
    // for its instructions.)
    auto for_each_4 = [&](auto f) {
#pragma unroll 1
        for (int i = w0 + 4 * lane; i - 4 * lane < w1; i += 128) {
            uint32_t k[4];
            if (kept) {
                const uint4 v = *reinterpret_cast<const uint4*>(keys + i - p0);
                k[0] = v.x; k[1] = v.y; k[2] = v.z; k[3] = v.w;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) k[e] = key_of(i + e);
            }
            f(i, k);
        }
    };
    uint32_t want = static_cast<uint32_t>(budget - recent);      // < old, since budget < len
    const bool any_old = want > 0;
    uint32_t prefix = 0, mask = 0;
    for (int i = tid; i < 2 * kEvBins; i += kEvThreads) hist[i] = 0;
    __syncthreads();
    if (any_old) {
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0);
            const uint32_t bins = pass == 2 ? 1024u : 2048u;
            uint32_t* h = hist + (pass & 1) * kEvBins;
            for_each_4([&](int, const uint32_t (&k)[4]) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if ((k[e] & mask) == prefix) atomicAdd(&h[(k[e] >> shift) & (bins - 1u)], 1u);
            });
            __syncthreads();
            const uint2 two = *reinterpret_cast<const uint2*>(h + 2 * tid);          // a warp's 64 bins together
            const uint32_t all = __reduce_add_sync(0xFFFFFFFFu, two.x + two.y);
            if (lane == 0) coarse[pass & 1][warp] = all;
            sync_all();
            // (every CTA has read the counts of the pass before by now)
            if (pass == 1) *reinterpret_cast<uint2*>(hist + 2 * tid) = make_uint2(0, 0);
            // one warp adds up the CTAs' counts, from the top bin down: the 64 bins in which they reach `want`, then the bin
            if (warp == 0) {
                const uint32_t at = smem_u32(&coarse[pass & 1][31 - lane]);
                uint32_t n = 0;
#pragma unroll
                for (int r = 0; r < CTAS; ++r) n += ld_cluster_u32(map_to_cta(at, r));
                uint32_t upto = warp_scan(n, lane);
                int who = __ffs(__ballot_sync(0xFFFFFFFFu, upto >= want)) - 1;
                const uint32_t left = want - __shfl_sync(0xFFFFFFFFu, upto - n, who);
                const int top = 64 * (31 - who) + 63 - 2 * lane;             // this lane's bins: top and top - 1
                const uint32_t at2 = smem_u32(h + top - 1);
                uint32_t c0 = 0, c1 = 0;
#pragma unroll
                for (int r = 0; r < CTAS; ++r) {
                    const uint2 v = ld_cluster_v2(map_to_cta(at2, r));
                    c0 += v.y; c1 += v.x;
                }
                upto = warp_scan(c0 + c1, lane);
                who = __ffs(__ballot_sync(0xFFFFFFFFu, upto >= left)) - 1;
                if (lane == who) {
                    const uint32_t before = upto - (c0 + c1);
                    const bool second = before + c0 < left;
                    s_bin = top - (second ? 1 : 0);
                    s_left = left - before - (second ? c0 : 0u);
                }
            }
            __syncthreads();
            prefix |= s_bin << shift;
            mask |= (bins - 1u) << shift;
            want = s_left;                           // (the next write of s_bin is two barriers away)
        }
    }
    // `want` of the positions with key == prefix stay, the lowest first
    auto is_sure = [&](int i, uint32_t k) { return i < w1 && (i >= old || (any_old && k > prefix)); };
    auto is_border = [&](int i, uint32_t k) { return any_old && i < w1_old && k == prefix; };
    uint32_t n_sure = 0, n_border = 0;
    for_each_4([&](int i, const uint32_t (&k)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            n_sure += is_sure(i + e, k[e]) ? 1u : 0u;
            n_border += is_border(i + e, k[e]) ? 1u : 0u;
        }
    });
    n_sure = __reduce_add_sync(0xFFFFFFFFu, n_sure);
    n_border = __reduce_add_sync(0xFFFFFFFFu, n_border);
    if (lane == 0) warp_count[warp] = make_uint2(n_sure, n_border);
    __syncthreads();
    const uint2 others = warp_count[lane];
    uint32_t sure_at = __reduce_add_sync(0xFFFFFFFFu, lane < warp ? others.x : 0u), border_at = __reduce_add_sync(0xFFFFFFFFu, lane < warp ? others.y : 0u);
    if (CTAS > 1) {
        if (warp == 0) {
            const uint32_t x = __reduce_add_sync(0xFFFFFFFFu, others.x), y = __reduce_add_sync(0xFFFFFFFFu, others.y);
            if (lane == 0) cta_count = make_uint2(x, y);
        }
        sync_all();
        uint2 v = make_uint2(0, 0);
        if (lane < rank) v = ld_cluster_v2(map_to_cta(smem_u32(&cta_count), lane));
        sure_at += __reduce_add_sync(0xFFFFFFFFu, v.x);
        border_at += __reduce_add_sync(0xFFFFFFFFu, v.y);
    }
    // (nearly every warp) its border positions go the same way, or they are told apart one by one
    const bool alike = n_border == 0 || border_at >= want || border_at + n_border <= want, too = border_at < want;
    const uint32_t below = (1u << lane) - 1u;
    uint32_t place = sure_at + min(border_at, want);
    for_each_4([&](int i, const uint32_t (&k)[4]) {
        bool stays[4];
        if (alike) {
#pragma unroll
            for (int e = 0; e < 4; ++e) stays[e] = is_sure(i + e, k[e]) || (too && is_border(i + e, k[e]));
        } else {
            uint32_t at = border_at;
            bool border[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                border[e] = is_border(i + e, k[e]);
                const uint32_t who = __ballot_sync(0xFFFFFFFFu, border[e]);
                at += __popc(who & below);
                border_at += __popc(who);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                stays[e] = is_sure(i + e, k[e]) || (border[e] && at < want);
                at += border[e] ? 1u : 0u;
            }
        }
        uint32_t at = place;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t who = __ballot_sync(0xFFFFFFFFu, stays[e]);
            at += __popc(who & below);
            place += __popc(who);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (stays[e]) out[at++] = i + e;
    });
    if (CTAS > 1) sync_all();                        // no CTA leaves while another may still read its counts
}

}  // namespace

template <int CTAS>
static cudaError_t launch_as(const float* acc, int64_t ld, const int32_t* lens, int B, int budget, int recent, int32_t* keep, int32_t* new_lens,
                             cudaStream_t stream) {
    const void* kernel = reinterpret_cast<const void*>(evict_select_kernel<CTAS>);
    if (cudaError_t e = ensure_max_dynamic_smem(kernel, kEvHistBytes + kEvKeys * 4); e != cudaSuccess) return e;
    // room for the longest slice that ld allows
    const int64_t slice = ((ld + CTAS - 1) / CTAS + 127) & ~int64_t(127);
    const int slots = static_cast<int>(slice < kEvKeys ? slice : kEvKeys);
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(B) * CTAS);
    cfg.blockDim = dim3(kEvThreads);
    cfg.dynamicSmemBytes = kEvHistBytes + static_cast<size_t>(slots) * 4;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CTAS;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = CTAS > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, evict_select_kernel<CTAS>, acc, ld, lens, budget, recent, slots, keep, new_lens);
}

// One CTA a sequence or a cluster of eight. A cluster costs about 4 us more to start and sweeps eight times as fast, but few clusters run at a time.
// Measured (us, one CTA | cluster; B sequences of ld positions, a quarter kept):
//   ld       B = 1         24            54            148           149
//   8192     8.3 |  8.5    8.4 | 11.0    8.4 | 20.8    8.6 | 49.3   13.9 | 49.6
//   16384   12.5 |  8.7   12.6 | 12.0   12.7 | 23.1   12.9 | 53.6   22.1 | 53.9
//   49152   29.0 | 10.9   29.5 | 15.8   29.5 | 30.5   29.7 | 71.6   56.9 | 72.2
//   65536   61.1 | 11.6   61.8 | 19.4   61.9 | 36.0   62.1 | 81.4  121.7 | 82.2      (the keys no longer fit one CTA's shared memory)
//   131072   117 | 16.0    118 | 29.6    118 | 52.4    127 | 124     236 | 125
// The border rises by about 512 positions with every sequence that runs at the same time as the others.
static bool one_cta_each(int64_t ld, int B) {
    const int waves = (B + 147) / 148;
    return ld <= 8192 + 512 * static_cast<int64_t>(B / waves);
}

cudaError_t launch_evict_select(const float* acc, int64_t ld, const int32_t* lens, int B, int budget, int recent, int32_t* keep,
                                int32_t* new_lens, cudaStream_t stream) {
    return one_cta_each(ld, B) ? launch_as<1>(acc, ld, lens, B, budget, recent, keep, new_lens, stream)
                               : launch_as<kEvCtas>(acc, ld, lens, B, budget, recent, keep, new_lens, stream);
}

}  // namespace idxc
