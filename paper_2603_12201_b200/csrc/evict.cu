// Which cached positions of a sequence stay when its cache is cut to a budget: the newest `recent` ones, and among the older
// ones the budget - recent with the largest accumulated attention weight (ties: lowest position), in ascending order.
// A cluster of eight CTAs takes a sequence, each an eighth of its positions, whose keys stay in shared memory (up to 48K positions a
// CTA; longer slices are read from global memory again). Three histogram passes (11 + 11 + 10 bits of an order-preserving key) find the
// key of the last position that stays exactly; the CTAs add up their histograms through distributed shared memory. Then every
// position's place in the output is the number of positions before it that stay, by prefix sums over lanes, warps and CTAs: no
// atomics on the output, ascending order for free. Bound by latency (eight cluster barriers and sweeps of a few microseconds, 25 us at
// 131072 positions), not by its bytes; one CTA per sequence took 313 us.
#include "kernels.h"
#include "ptx_sm100.cuh"

namespace idxc {
namespace {

constexpr int kEvCtas = 8;                           // CTAs of a long sequence (short ones, up to kEvShort positions a row of acc: one)
constexpr int kEvShort = 16384;
constexpr int kEvThreads = 1024;
constexpr int kEvWarps = kEvThreads / 32;
constexpr int kEvBins = 2 * kEvThreads;               // 2048, two a thread
constexpr int kEvKeys = 49152;                       // keys of a slice that fit into shared memory at most
constexpr uint32_t kEvHistBytes = 2 * kEvBins * 4;

// Larger float = larger key; -0 and +0 share a key.
__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ uint2 ld_cluster_v2(uint32_t addr) {
    uint2 v;
    asm volatile("ld.shared::cluster.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
    return v;
}

template <int CTAS>
__global__ void __launch_bounds__(kEvThreads)
evict_select_kernel(const float* __restrict__ acc, int64_t ld, const int32_t* __restrict__ lens, int budget, int recent, int key_slots,
                    int32_t* __restrict__ keep, int32_t* __restrict__ new_lens) {
    extern __shared__ __align__(16) uint32_t ev_smem[];
    uint32_t* hist = ev_smem;                        // [2][kEvBins]
    uint32_t* keys = ev_smem + 2 * kEvBins;          // [key_slots]
    __shared__ uint32_t warp_sum[kEvWarps];
    __shared__ uint2 warp_count[kEvWarps];
    __shared__ uint32_t s_bin, s_left;
    __shared__ __align__(8) uint2 cta_count;         // positions of this CTA that certainly stay, and those at the border key
    auto sync_all = [&]() {                          // the CTAs of the sequence
        if (CTAS > 1) cluster_sync();
        else __syncthreads();
    };
    const int rank = CTAS > 1 ? static_cast<int>(cluster_ctarank()) : 0;
    const int b = blockIdx.x / CTAS, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int len = static_cast<int>(min(static_cast<int64_t>(max(__ldg(lens + b), 0)), ld));
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
    const int slice = ((len + CTAS - 1) / CTAS + 31) & ~31;
    const int p0 = min(rank * slice, len), p1 = min(p0 + slice, len);
    const int p1_old = min(p1, old);
    const bool kept = slice <= key_slots;
    if (kept)
        for (int i = p0 + tid; i < p1_old; i += kEvThreads) keys[i - p0] = order_key(__ldg(row + i));
    auto key_at = [&](int i) -> uint32_t { return kept ? keys[i - p0] : order_key(__ldg(row + i)); };
    uint32_t want = static_cast<uint32_t>(budget - recent);      // < old, since budget < len
    const bool any_old = want > 0;
    uint32_t prefix = 0, mask = 0;
    for (int i = tid; i < kEvBins; i += kEvThreads) hist[i] = 0;
    __syncthreads();
    if (any_old) {
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0);
            const uint32_t bins = pass == 2 ? 1024u : 2048u;
            uint32_t* h = hist + (pass & 1) * kEvBins;
            for (int i = p0 + tid; i < p1_old; i += kEvThreads) {
                const uint32_t k = key_at(i);
                if ((k & mask) == prefix) atomicAdd(&h[(k >> shift) & (bins - 1u)], 1u);
            }
            sync_all();
            // (every CTA has read the other buffer by now: it may be cleared for the next pass)
            for (int i = tid; i < kEvBins; i += kEvThreads) hist[((pass + 1) & 1) * kEvBins + i] = 0;
            // counts of all CTAs from the top bin down: the bin in which they reach `want`. Thread t has bins top and top - 1.
            const int top = kEvBins - 1 - 2 * tid;
            const uint32_t at = smem_u32(h + top - 1);
            uint32_t c[2] = {0, 0};
#pragma unroll
            for (int r = 0; r < CTAS; ++r) {
                const uint2 v = ld_cluster_v2(map_to_cta(at, r));
                c[0] += v.y; c[1] += v.x;
            }
            const uint32_t mine = c[0] + c[1];
            uint32_t run = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t y = __shfl_up_sync(0xFFFFFFFFu, run, o);
                if (lane >= o) run += y;
            }
            if (lane == 31) warp_sum[warp] = run;
            __syncthreads();
            uint32_t before = run - mine;
            for (int w = 0; w < warp; ++w) before += warp_sum[w];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (before < want && before + c[j] >= want) { s_bin = top - j; s_left = want - before; }
                before += c[j];
            }
            __syncthreads();
            prefix |= s_bin << shift;
            mask |= (bins - 1u) << shift;
            want = s_left;
            __syncthreads();
        }
    }
    // `want` of the positions with key == prefix stay, the lowest first. A warp has a run of its CTA's slice.
    const int seg = (((slice + kEvWarps - 1) / kEvWarps) + 31) & ~31;
    const int w0 = min(p0 + warp * seg, p1), w1 = min(w0 + seg, p1);
    auto look = [&](int i, bool& sure, bool& border) {
        sure = i >= old && i < w1;
        border = false;
        if (any_old && i < old && i < w1) {
            const uint32_t k = key_at(i);
            sure = k > prefix;
            border = k == prefix;
        }
    };
    uint32_t n_sure = 0, n_border = 0;
    for (int i0 = w0; i0 < w1; i0 += 32) {
        bool sure, border;
        look(i0 + lane, sure, border);
        n_sure += __popc(__ballot_sync(0xFFFFFFFFu, sure));
        n_border += __popc(__ballot_sync(0xFFFFFFFFu, border));
    }
    if (lane == 0) warp_count[warp] = make_uint2(n_sure, n_border);
    __syncthreads();
    uint32_t sure_at = 0, border_at = 0;
    for (int w = 0; w < kEvWarps; ++w) {
        const uint2 v = warp_count[w];
        if (w < warp) { sure_at += v.x; border_at += v.y; }
        if (tid == 0) { n_sure = w == 0 ? v.x : n_sure + v.x; n_border = w == 0 ? v.y : n_border + v.y; }
    }
    if (tid == 0) cta_count = make_uint2(n_sure, n_border);
    sync_all();
    for (int r = 0; r < rank; ++r) {
        const uint2 v = ld_cluster_v2(map_to_cta(smem_u32(&cta_count), r));
        sure_at += v.x;
        border_at += v.y;
    }
    for (int i0 = w0; i0 < w1; i0 += 32) {
        bool sure, border;
        look(i0 + lane, sure, border);
        const uint32_t bs = __ballot_sync(0xFFFFFFFFu, sure), bb = __ballot_sync(0xFFFFFFFFu, border), below = (1u << lane) - 1u;
        const uint32_t my_sure = sure_at + __popc(bs & below), my_border = border_at + __popc(bb & below);
        const uint32_t place = my_sure + min(my_border, want);
        if ((sure || (border && my_border < want)) && place < static_cast<uint32_t>(budget)) out[place] = i0 + lane;
        sure_at += __popc(bs);
        border_at += __popc(bb);
    }
    sync_all();                                  // no CTA leaves while another may still read its counts
}

}  // namespace

template <int CTAS>
static cudaError_t launch_as(const float* acc, int64_t ld, const int32_t* lens, int B, int budget, int recent, int32_t* keep, int32_t* new_lens,
                             cudaStream_t stream) {
    const void* kernel = reinterpret_cast<const void*>(evict_select_kernel<CTAS>);
    if (cudaError_t e = ensure_max_dynamic_smem(kernel, kEvHistBytes + kEvKeys * 4); e != cudaSuccess) return e;
    // room for the longest slice that ld allows: short rows leave room for several CTAs on an SM
    const int64_t slice = ((ld + CTAS - 1) / CTAS + 31) & ~int64_t(31);
    const int slots = static_cast<int>(slice < kEvKeys ? slice : kEvKeys);
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(B) * CTAS);
    cfg.blockDim = dim3(kEvThreads);
    cfg.dynamicSmemBytes = kEvHistBytes + static_cast<size_t>(slots) * 4;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = CTAS;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = CTAS > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, evict_select_kernel<CTAS>, acc, ld, lens, budget, recent, slots, keep, new_lens);
}

cudaError_t launch_evict_select(const float* acc, int64_t ld, const int32_t* lens, int B, int budget, int recent, int32_t* keep,
                                int32_t* new_lens, cudaStream_t stream) {
    return ld <= kEvShort ? launch_as<1>(acc, ld, lens, B, budget, recent, keep, new_lens, stream)
                          : launch_as<kEvCtas>(acc, ld, lens, B, budget, recent, keep, new_lens, stream);
}

}  // namespace idxc
