// Writing and reading rows of a paged key/value cache, and the bounds of its pages: for every page, head and key column the smallest and the
// largest value among the rows 0 .. (newest written), as the rows read back in bf16.
//
// Append. Tokens that follow each other into one page are a run; the CTA that holds a run's first token walks the page's rows once: those in
// front of the run come from the cache, the run's from the input, and go to the cache on the way. So a page's bounds come from its rows alone
// (never from what they were), one thread owns a column's bounds, and nothing is read twice. A thread owns 8 columns (16 bytes) of a head; what
// a head's 8 or 16 threads share is only the row's maximum in front of the e4m3 codes. HBM-bound: 8 bytes moved per element of k and v in bf16
// (read, written), 6 in e4m3, and for a decode step the latency of one page's rows. Measured: 70299 tokens of 8 heads with d = 128 in e4m3 105 us (4.1 TB/s
// of what is read and written; bound by its instructions, 75 % of the issue slots), in bf16 97 us (5.9 TB/s), 32 tokens in bf16 6.2 us; the same read back 78 to 84, 88
// and 5 us. Few long pages leave most of the GPU idle: 1000 tokens of 8 heads, d = 128, bf16 / e4m3, take 7 / 10 us in pages of 16, 12 / 23 in pages of 64, and 89 / 255
// in one of 1024, which is one CTA's.
#include "e4m3_rows.cuh"
#include "kernels.h"
#include "ptx_sm100.cuh"

namespace idxc {
namespace {

constexpr int kAppendThreads = 256;

// Values of 8 e4m3 codes and their row's scale, rounded to bf16.
__device__ __forceinline__ uint4 codes_to_bf16(uint2 codes, float scale) {
    uint4 out;
    uint32_t* o = &out.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t two = (i < 2 ? codes.x : codes.y) >> (16 * (i & 1)) & 0xFFFFu;
        const uint32_t h = e4m3x2_to_f16x2(two);
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
        const __nv_bfloat162 v = __floats2bfloat162_rn(f.x * scale, f.y * scale);
        o[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
    return out;
}
__device__ __forceinline__ void widen(uint4 v, uint4& lo, uint4& hi) {
    const uint32_t* x = &v.x;
    uint32_t *l = &lo.x, *h = &hi.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 y = *reinterpret_cast<const __nv_bfloat162*>(x + i);
        __nv_bfloat162 a = __hmin2(*reinterpret_cast<__nv_bfloat162*>(l + i), y), b = __hmax2(*reinterpret_cast<__nv_bfloat162*>(h + i), y);
        l[i] = *reinterpret_cast<uint32_t*>(&a);
        h[i] = *reinterpret_cast<uint32_t*>(&b);
    }
}
constexpr uint32_t kBf16PosInf2 = 0x7F807F80u, kBf16NegInf2 = 0xFF80FF80u;

struct AppendArgs {
    PagedCache c;
    const uint4* k;              // rows of H_kv * d bf16, k_stride / v_stride vectors of 8 apart
    const uint4* v;
    int64_t k_stride, v_stride;
    const int64_t* slots;
    int64_t n;
    int chunk;                   // tokens a CTA looks at for the beginnings of runs: at most 32
};

// x / 448, correctly rounded (as div_by_scale; x normal and, but for an infinite one, below 2^128).
__device__ __forceinline__ float over_448(float x) { return x <= 3.4e38f ? div_by_scale(x, kE4m3Max, 1.f / kE4m3Max) : x; }
// Largest magnitudes of a key's and of a value's 8 elements, as two bf16 (a number that is none counts as 0).
__device__ __forceinline__ uint32_t two_maxima(uint4 k, uint4 v) {
    auto one = [](uint4 x) -> __nv_bfloat162 {
        auto abs2 = [](uint32_t w) -> __nv_bfloat162 {
            w &= 0x7FFF7FFFu;
            return *reinterpret_cast<const __nv_bfloat162*>(&w);
        };
        return __hmax2(__hmax2(abs2(x.x), abs2(x.y)), __hmax2(abs2(x.z), abs2(x.w)));
    };
    const __nv_bfloat162 a = one(k), b = one(v);
    const __nv_bfloat162 m = __hmax2(__lows2bfloat162(a, b), __highs2bfloat162(a, b));
    return *reinterpret_cast<const uint32_t*>(&m);
}

template <bool FP8, int D>
__global__ void __launch_bounds__(kAppendThreads, 3)
paged_append_kernel(const AppendArgs a) {
    __shared__ int run_len;
    __shared__ uint4 part[2][kAppendThreads];
    let_next_start();
    wait_for_previous();
    const PagedCache& c = a.c;
    constexpr int per_head = D / 8;
    const int vecs = c.H_kv * per_head;
    const int cols = min(vecs, kAppendThreads), lanes = kAppendThreads / cols;       // threads of a row, rows at a time
    const int lane = threadIdx.x / cols;
    const int col = blockIdx.y * kAppendThreads + threadIdx.x % cols;
    const bool works = lane < lanes && col < vecs;
    const int head = col / per_head, d0 = (col % per_head) * 8;
    const int64_t n_slots = c.n_pages * c.page_size;
    const int64_t t_end = min(a.n, (static_cast<int64_t>(blockIdx.x) + 1) * a.chunk);
    // Tokens of the chunk that begin a run: every warp finds them for itself.
    const int64_t t_first = static_cast<int64_t>(blockIdx.x) * a.chunk, t_mine = t_first + (threadIdx.x & 31);
    bool begins = false;
    if (t_mine < t_end) {
        const int64_t slot = a.slots[t_mine];
        begins = slot >= 0 && slot < n_slots && !(t_mine > 0 && slot % c.page_size != 0 && a.slots[t_mine - 1] == slot - 1);
    }
    for (uint32_t runs = __ballot_sync(0xFFFFFFFFu, begins); runs; runs &= runs - 1) {
        const int64_t t0 = t_first + (__ffs(runs) - 1);
        const int64_t slot = a.slots[t0], page = slot / c.page_size;
        const int off = static_cast<int>(slot - page * c.page_size);
        __syncthreads();
        if (threadIdx.x == 0) run_len = c.page_size - off;
        __syncthreads();
        for (int i = threadIdx.x; i < c.page_size - off; i += kAppendThreads)
            if (t0 + i >= a.n || a.slots[t0 + i] != slot + i) {
                atomicMin(&run_len, i);
                break;
            }
        __syncthreads();
        const int n_new = run_len, rows = off + n_new;
        uint4 lo = make_uint4(kBf16PosInf2, kBf16PosInf2, kBf16PosInf2, kBf16PosInf2);
        uint4 hi = make_uint4(kBf16NegInf2, kBf16NegInf2, kBf16NegInf2, kBf16NegInf2);
        const int64_t base = page * c.page_stride + head * c.head_stride + d0;        // elements
        const int64_t scale_base = (page * c.H_kv + head) * c.page_size;
        constexpr int U = 2, U_OLD = FP8 ? 2 : 4;                                               // rows of a thread on their way
        // new rows: the next U of a thread are on their way while these are worked on
        const uint4 *k_from = a.k + (t0 + lane) * a.k_stride + col, *v_from = a.v + (t0 + lane) * a.v_stride + col;
        const int64_t k_step = lanes * a.k_stride, v_step = lanes * a.v_stride, to_step = lanes * c.token_stride;
        int64_t to = base + (off + lane) * c.token_stride;
        uint4 k_next[U], v_next[U];
        auto fetch = [&](int i0) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool in = works && i0 + u * lanes + lane < n_new;
                k_next[u] = in ? *k_from : make_uint4(0u, 0u, 0u, 0u);
                v_next[u] = in ? *v_from : make_uint4(0u, 0u, 0u, 0u);
                k_from += k_step;
                v_from += v_step;
            }
        };
        fetch(0);
        if (c.bounds)
            for (int r0 = lane; r0 < off; r0 += U_OLD * lanes) {                          // rows that are there
                uint4 x[U_OLD];
#pragma unroll
                for (int u = 0; u < U_OLD; ++u) {
                    const int r = r0 + u * lanes;
                    if (!works || r >= off) continue;
                    const int64_t at = base + r * c.token_stride;
                    if (FP8)
                        x[u] = codes_to_bf16(*reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(c.k) + at), c.k_scale[scale_base + r]);
                    else
                        x[u] = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(c.k) + at);
                }
#pragma unroll
                for (int u = 0; u < U_OLD; ++u)
                    if (works && r0 + u * lanes < off) widen(x[u], lo, hi);
            }
        for (int i0 = 0; i0 < n_new; i0 += U * lanes) {                               // (all threads: they shuffle)
            Vec8 k[U], v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                k[u].raw = k_next[u];
                v[u].raw = v_next[u];
            }
            if (i0 + U * lanes < n_new) fetch(i0 + U * lanes);
#pragma unroll
            for (int u = 0; u < U; ++u, to += to_step) {
                const int i = i0 + u * lanes + lane;
                const bool in = works && i < n_new;
                if (!FP8) {
                    if (in) {
                        *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(c.k) + to) = k[u].raw;
                        *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(c.v) + to) = v[u].raw;
                        widen(k[u].raw, lo, hi);
                    }
                    continue;
                }
                uint32_t m = two_maxima(k[u].raw, v[u].raw);
#pragma unroll
                for (int o = per_head / 2; o > 0; o >>= 1) {                          // (a head's threads are aligned within a warp)
                    const uint32_t y = __shfl_xor_sync(0xFFFFFFFFu, m, o);
                    const __nv_bfloat162 z = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&m), *reinterpret_cast<const __nv_bfloat162*>(&y));
                    m = *reinterpret_cast<const uint32_t*>(&z);
                }
                const float k_max = __uint_as_float(m << 16), v_max = __uint_as_float(m & 0xFFFF0000u);
                if (in) {
                    const float ks = over_448(fmaxf(k_max, 1e-12f)), vs = over_448(fmaxf(v_max, 1e-12f));
                    const uint2 kc = quantize8(k[u], ks);
                    *reinterpret_cast<uint2*>(static_cast<uint8_t*>(c.k) + to) = kc;
                    *reinterpret_cast<uint2*>(static_cast<uint8_t*>(c.v) + to) = quantize8(v[u], vs);
                    if (d0 == 0) {
                        c.k_scale[scale_base + off + i] = ks;
                        c.v_scale[scale_base + off + i] = vs;
                    }
                    if (c.bounds) widen(codes_to_bf16(kc, ks), lo, hi);
                }
            }
        }
        if (!c.bounds) continue;
        if (lanes > 1) {                                                              // columns meet from the rows that went side by side
            part[0][threadIdx.x] = lo;
            part[1][threadIdx.x] = hi;
            __syncthreads();
            if (lane == 0)
                for (int l = 1; l < lanes; ++l) {
                    uint4 dummy = hi;
                    widen(part[0][l * cols + threadIdx.x], lo, dummy);
                    dummy = lo;
                    widen(part[1][l * cols + threadIdx.x], dummy, hi);
                }
        }
        if (works && lane == 0 && rows > 0) {
            __nv_bfloat16* edge = static_cast<__nv_bfloat16*>(c.bounds) + (page * c.H_kv + head) * 2 * D + d0;
            *reinterpret_cast<uint4*>(edge) = lo;
            *reinterpret_cast<uint4*>(edge + D) = hi;
        }
    }
}

// Division of numbers below 2^31 by a number that is known on the host, by a product (T. Granlund and P. Montgomery, Division by invariant integers using
// multiplication, 1994): with 2^(l-1) < d <= 2^l and m = floor(2^32 (2^l - d) / d) + 1 the quotient is (n + floor(m n / 2^32)) >> l.
struct Divisor {
    unsigned m, l;
    explicit Divisor(unsigned d) : l(0) {
        while ((1ull << l) < d) ++l;
        m = static_cast<unsigned>((((1ull << l) - d) << 32) / d + 1);
    }
    __device__ __forceinline__ unsigned operator()(unsigned n) const { return (n + __umulhi(m, n)) >> l; }
};

// Rows of the cache in bf16; slots outside the cache give zeros. A CTA writes kGatherVecs neighbouring 16-byte vectors of each output, a thread
// four of each, whose loads are on their way together. (Vectors a grid apart instead of 256: 112 us instead of 80 for 70299 rows of 8 heads in 8 bits.)
constexpr int kGatherVecs = 1024;
template <bool FP8, int D>
__global__ void __launch_bounds__(256)
paged_gather_kernel(const PagedCache c, const Divisor by_vecs, const Divisor by_page, const int64_t* slots, int64_t n, uint4* k_out, uint4* v_out) {
    let_next_start();
    wait_for_previous();
    constexpr unsigned per_head = D / 8;
    const unsigned vecs = c.H_kv * per_head;
    const int64_t n_slots = c.n_pages * c.page_size, first = blockIdx.x * int64_t(kGatherVecs), all = n * vecs;
    const int64_t t_first = first / vecs;
    const unsigned rest = static_cast<unsigned>(first - t_first * vecs);
    constexpr int U = kGatherVecs / 256;
    uint4 k[U], v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const unsigned i = u * 256 + threadIdx.x;
        k[u] = v[u] = make_uint4(0u, 0u, 0u, 0u);
        if (first + i >= all) continue;
        const unsigned t = by_vecs(rest + i), col = rest + i - t * vecs, head = col / per_head, d0 = (col - head * per_head) * 8;
        const int64_t slot = slots[t_first + t];
        if (slot < 0 || slot >= n_slots) continue;
        const unsigned page = by_page(static_cast<unsigned>(slot)), off = static_cast<unsigned>(slot) - page * c.page_size;
        const int64_t at = page * c.page_stride + off * c.token_stride + head * c.head_stride + d0;
        if (FP8) {
            const int64_t s = (static_cast<int64_t>(page) * c.H_kv + head) * c.page_size + off;
            k[u] = codes_to_bf16(*reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(c.k) + at), c.k_scale[s]);
            v[u] = codes_to_bf16(*reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(c.v) + at), c.v_scale[s]);
        } else {
            k[u] = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(c.k) + at);
            v[u] = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(c.v) + at);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t i = first + u * 256 + threadIdx.x;
        if (i < all) {
            k_out[i] = k[u];
            v_out[i] = v[u];
        }
    }
}

}  // namespace

cudaError_t launch_paged_append(const PagedCache& c, const void* k, int64_t k_stride, const void* v, int64_t v_stride, const int64_t* slots, int64_t n,
                                cudaStream_t stream) {
    // A CTA for every token as long as that fills the GPU a few times over (a decode step's pages then go side by side); longer inputs are
    // prompts, whose runs are as long as pages.
    const int chunk = n <= 4096 ? 1 : 16;
    const AppendArgs a{c, static_cast<const uint4*>(k), static_cast<const uint4*>(v), k_stride / 8, v_stride / 8, slots, n, chunk};
    const int vecs = c.H_kv * (c.d / 8);
    const dim3 grid(static_cast<unsigned>((n + chunk - 1) / chunk), static_cast<unsigned>((vecs + kAppendThreads - 1) / kAppendThreads));
    if (c.d == 128)
        return c.fp8 ? launch_behind(paged_append_kernel<true, 128>, grid, kAppendThreads, 0, stream, a)
                     : launch_behind(paged_append_kernel<false, 128>, grid, kAppendThreads, 0, stream, a);
    return c.fp8 ? launch_behind(paged_append_kernel<true, 64>, grid, kAppendThreads, 0, stream, a)
                 : launch_behind(paged_append_kernel<false, 64>, grid, kAppendThreads, 0, stream, a);
}

cudaError_t launch_paged_gather(const PagedCache& c, const int64_t* slots, int64_t n, void* k_out, void* v_out, cudaStream_t stream) {
    const unsigned grid = static_cast<unsigned>((n * c.H_kv * (c.d / 8) + kGatherVecs - 1) / kGatherVecs);
    auto go = [&](auto kernel) {
        return launch_behind(kernel, dim3(grid), 256, 0, stream, c, Divisor(c.H_kv * (c.d / 8)), Divisor(c.page_size), slots, n, static_cast<uint4*>(k_out),
                             static_cast<uint4*>(v_out));
    };
    if (c.d == 128) return c.fp8 ? go(paged_gather_kernel<true, 128>) : go(paged_gather_kernel<false, 128>);
    return c.fp8 ? go(paged_gather_kernel<true, 64>) : go(paged_gather_kernel<false, 64>);
}

}  // namespace idxc
