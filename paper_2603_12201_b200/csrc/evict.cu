// Which cached positions of a sequence stay when its cache is cut to a budget: the newest `recent` ones, and among the older
// ones the budget - recent with the largest accumulated attention weight (ties: lowest position), in ascending order.
// One CTA per sequence: three histogram passes (11 + 11 + 10 bits of an order-preserving key) find the weight of the last
// one that stays exactly, and one ordered pass writes the positions.
#include "kernels.h"

namespace idxc {
namespace {

constexpr int kEvThreads = 1024;
constexpr int kEvBins = 2048;

// Larger float = larger key; -0 and +0 share a key.
__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__global__ void __launch_bounds__(kEvThreads)
evict_select_kernel(const float* __restrict__ acc, int64_t ld, const int32_t* __restrict__ lens, int budget, int recent,
                    int32_t* __restrict__ keep, int32_t* __restrict__ new_lens) {
    __shared__ uint32_t hist[kEvBins];
    __shared__ uint32_t warp_sum[kEvThreads / 32];
    __shared__ uint32_t s_bin, s_left;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int len = static_cast<int>(min(static_cast<int64_t>(max(__ldg(lens + b), 0)), ld));
    const float* row = acc + b * ld;
    int32_t* out = keep + static_cast<int64_t>(b) * budget;
    const int stay = min(len, budget);
    if (tid == 0) new_lens[b] = stay;
    for (int j = stay + tid; j < budget; j += kEvThreads) out[j] = -1;
    if (len <= budget) {
        for (int j = tid; j < len; j += kEvThreads) out[j] = j;
        return;
    }
    const int old = len - recent;                 // positions that compete
    uint32_t want = static_cast<uint32_t>(budget - recent);      // < old, since budget < len
    uint32_t prefix = 0, mask = 0;
    if (want > 0) {
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0);
            const int bins = pass == 2 ? 1024 : 2048;
            for (int i = tid; i < kEvBins; i += kEvThreads) hist[i] = 0;
            __syncthreads();
            for (int i = tid; i < old; i += kEvThreads) {
                const uint32_t k = order_key(__ldg(row + i));
                if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & (bins - 1)], 1u);
            }
            __syncthreads();
            // from the top bin down: the bin in which the count reaches `want`; thread t holds the two bins below the top 2t
            const int hi = kEvBins - 1 - 2 * tid;
            const uint32_t c0 = hist[hi], c1 = hist[hi - 1];
            uint32_t run = c0 + c1;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t y = __shfl_up_sync(0xFFFFFFFFu, run, o);
                if (lane >= o) run += y;
            }
            if (lane == 31) warp_sum[warp] = run;
            __syncthreads();
            uint32_t before = run - c0 - c1;
            for (int w = 0; w < warp; ++w) before += warp_sum[w];
            if (before < want && before + c0 >= want) { s_bin = hi; s_left = want - before; }
            else if (before + c0 < want && before + c0 + c1 >= want) { s_bin = hi - 1; s_left = want - before - c0; }
            __syncthreads();
            prefix |= s_bin << shift;
            mask |= static_cast<uint32_t>(bins - 1) << shift;
            want = s_left;
            __syncthreads();
        }
    }
    // `want` of the positions with key == prefix stay, the lowest first
    uint32_t n_out = 0, n_equal = 0;
    const bool any_old = budget > recent;
    for (int i0 = 0; i0 < len; i0 += kEvThreads) {
        const int i = i0 + tid;
        uint32_t k = 0;
        bool eq = false, above = false;
        if (i < old && any_old) {
            k = order_key(__ldg(row + i));
            eq = k == prefix;
            above = k > prefix;
        }
        const bool rec = i >= old && i < len;
        const uint32_t be = __ballot_sync(0xFFFFFFFFu, eq);
        if (lane == 0) warp_sum[warp] = __popc(be);
        __syncthreads();
        uint32_t eq_before = n_equal, eq_all = 0;
        for (int w = 0; w < kEvThreads / 32; ++w) {
            if (w < warp) eq_before += warp_sum[w];
            eq_all += warp_sum[w];
        }
        eq_before += __popc(be & ((1u << lane) - 1u));
        __syncthreads();
        const bool sel = rec || above || (eq && eq_before < want);
        const uint32_t bs = __ballot_sync(0xFFFFFFFFu, sel);
        if (lane == 0) warp_sum[warp] = __popc(bs);
        __syncthreads();
        uint32_t pos = n_out, all = 0;
        for (int w = 0; w < kEvThreads / 32; ++w) {
            if (w < warp) pos += warp_sum[w];
            all += warp_sum[w];
        }
        pos += __popc(bs & ((1u << lane) - 1u));
        if (sel && pos < static_cast<uint32_t>(budget)) out[pos] = i;
        n_out += all;
        n_equal += eq_all;
        __syncthreads();
    }
}

}  // namespace

cudaError_t launch_evict_select(const float* acc, int64_t ld, const int32_t* lens, int B, int budget, int recent, int32_t* keep,
                                int32_t* new_lens, cudaStream_t stream) {
    evict_select_kernel<<<static_cast<unsigned>(B), kEvThreads, 0, stream>>>(acc, ld, lens, budget, recent, keep, new_lens);
    return cudaGetLastError();
}

}  // namespace idxc
