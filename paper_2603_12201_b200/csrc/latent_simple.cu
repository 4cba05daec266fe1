// Head-summed attention weights over a latent cache, plain CUDA-core form.
#include "kernels.h"
#include "latent_format.cuh"

namespace idxc {
namespace {

constexpr int kPer = kLatentCols / 32;    // columns of a lane

// Column lane + 32 i of a cache row, i < 18, as floats.
__device__ __forceinline__ void read_row(const uint8_t* kv, bool q4, int64_t row, int lane, float (&v)[kPer]) {
    if (!q4) {
        const __nv_bfloat16* p = reinterpret_cast<const __nv_bfloat16*>(kv + row * kLatentBf16RowBytes);
#pragma unroll
        for (int i = 0; i < kPer; ++i) v[i] = __bfloat162float(p[lane + 32 * i]);
        return;
    }
    const uint8_t* p = kv + row * kLatentQ4RowBytes;
    const __nv_bfloat16* s = reinterpret_cast<const __nv_bfloat16*>(p + kLatentQ4ScaleOff);
    const __nv_bfloat16* r = reinterpret_cast<const __nv_bfloat16*>(p + kLatentQ4RopeOff);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int c = lane + 32 * i, e = c & 7, nibble = (e & 1) * 4 + (e >> 1);
        const uint32_t word = reinterpret_cast<const uint32_t*>(p)[c >> 3];
        v[i] = static_cast<float>(static_cast<int>((word >> (4 * nibble)) & 15u) - 8) * __bfloat162float(s[i]);
    }
    v[16] = __bfloat162float(r[lane]);
    v[17] = __bfloat162float(r[lane + 32]);
}

__device__ __forceinline__ int64_t cache_row(const LatentArgs& a, int b, int64_t j) {
    const int64_t base = a.kv_base ? a.kv_base[b] : 0;
    int64_t r = j;
    if (a.topk) {
        r = a.topk[static_cast<int64_t>(b) * a.k_top + j];
        if (r < 0) return -1;
    }
    r += base;
    return r >= 0 && r < a.n_kv ? r : -1;
}

__device__ __forceinline__ int64_t entries(const LatentArgs& a, int b) {
    if (a.topk) return a.k_top;
    const int64_t n = a.lens[b];
    return n < 0 ? 0 : (n > a.max_len ? a.max_len : n);
}

// One warp per position: its probability under every query row, summed.
__global__ void __launch_bounds__(256)
attn_weights_simple_kernel(const LatentArgs a, const float* __restrict__ lse, float beta, float* __restrict__ acc, int64_t ld) {
    const int b = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rows = a.n_step * a.H;
    const int64_t n = entries(a, b);
    const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.q) + static_cast<int64_t>(b) * rows * kLatentCols;
    for (int64_t j = static_cast<int64_t>(blockIdx.y) * 8 + warp; j < n; j += static_cast<int64_t>(gridDim.y) * 8) {
        const int64_t row = cache_row(a, b, j);
        float sum = 0.f;
        if (row >= 0) {
            float v[kPer];
            read_row(static_cast<const uint8_t*>(a.kv), a.q4 != 0, row, lane, v);
            for (int r = 0; r < rows; ++r) {
                float x = 0.f;
#pragma unroll
                for (int i = 0; i < kPer; ++i) x += __bfloat162float(q[static_cast<int64_t>(r) * kLatentCols + lane + 32 * i]) * v[i];
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
                const float s = lse[static_cast<int64_t>(b) * rows + r];
                const bool seen = a.topk || j < n - (a.n_step - 1 - r / a.H);
                if (seen && s > -INFINITY) sum += expf(x * a.scale - s);
            }
        }
        if (lane != 0) continue;
        if (!a.topk) {
            float* dst = acc + b * ld + j;
            *dst = (beta == 0.f ? 0.f : beta * *dst) + sum;
        } else if (row >= 0) {
            const int64_t s = a.topk[static_cast<int64_t>(b) * a.k_top + j];
            if (s < ld) atomicAdd(acc + b * ld + s, sum);
        }
    }
}

}  // namespace

cudaError_t launch_attn_weights(const LatentArgs& a, const float* lse, float beta, float* acc, int64_t ld, cudaStream_t stream) {
    const int64_t n = a.topk ? a.k_top : a.max_len;
    int64_t blocks = (n + 7) / 8;
    if (blocks > 2048) blocks = 2048;
    attn_weights_simple_kernel<<<dim3(static_cast<unsigned>(a.B), static_cast<unsigned>(blocks)), 256, 0, stream>>>(a, lse, beta, acc, ld);
    return cudaGetLastError();
}

}  // namespace idxc
