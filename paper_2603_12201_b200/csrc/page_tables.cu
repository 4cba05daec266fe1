// Block tables and slot maps of a paged cache, built on the GPU from the requests' lengths. With P = page size, a request of len
// positions owns ceil(len / P) pages; the free pages are a stack.
//     pages for n_b new tokens:  need_b = ceil((len_b + n_b) / P) - ceil(len_b / P); in flat order i over requests and their new pages the
//                                page is free[count - 1 - i]
//     slot of a position:        table[b][position / P] * P + position % P
// Giving pages back enters them in the reverse of that order, so that it undoes the taking (entries that are no page stay off the stack). All of it is a scan over the requests and
// then one independent load and store an entry: a few microseconds of latency, no bandwidth to speak of. The scan is one CTA's (requests
// in blocks of 1024), which also enters the pages and, for a decode step, the slots; the slots of many tokens are a second kernel's, with a
// token a thread, which finds its request by bisection. Measured (caches cold): 256 requests with 4 tokens each 7 us, giving back 5, positions to rows
// 4.5 for 256 x 2048; slots of 111489 tokens 4.4.
#include <type_traits>

#include "kernels.h"
#include "ptx_sm100.cuh"

namespace idxc {
namespace {

constexpr int kThreads = 1024;
constexpr int64_t kNever = int64_t(1) << 40;      // need of a request that cannot be served: it and all behind it are refused
// Table entries of a thread where 1024 requests give back more than one each. (102400 pages of 1024 requests 82 us, with 8 a thread 137; 1680 of 24
// requests 12.6 us with the calls around it, 14.1 with 8.)
constexpr int kGiveBack = 4;
constexpr int kFewTokens = 8192;                  // slots that the scanning CTA writes itself

__device__ __forceinline__ int64_t warp_scan(int64_t v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xFFFFFFFFu, v, o);
        if (lane >= o) v += y;
    }
    return v;
}
// Inclusive sums over the CTA; `all` receives the total. scratch: 32 words of shared memory.
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t* scratch, int64_t& all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t incl = warp_scan(v);
    __syncthreads();
    if (lane == 31) scratch[warp] = incl;
    __syncthreads();
    const int64_t sums = warp_scan(scratch[lane]);
    all = __shfl_sync(0xFFFFFFFFu, sums, 31);
    const int64_t before = __shfl_sync(0xFFFFFFFFu, sums, warp > 0 ? warp - 1 : 0);
    return warp > 0 ? incl + before : incl;
}
// The last r of the ascending first[0 .. n - 1] with first[r] <= i.
template <typename T>
__device__ __forceinline__ int find_last(const T* first, int n, T i) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= i) lo = mid;
        else hi = mid;
    }
    return lo;
}
__device__ __forceinline__ int pages_of(unsigned n, unsigned P) { return static_cast<int>((n + P - 1) / P); }      // n below 2^31

__global__ void __launch_bounds__(kThreads)
page_tables_kernel(int32_t* table, int64_t ld, int32_t* lens, const int32_t* new_tokens, int B, int P, const int32_t* free_pages,
                   int64_t free_cap, int32_t* free_count, int32_t* token_begin, int32_t* start, int64_t* slots, int64_t n_slots, int32_t* seq,
                   bool write_slots) {
    __shared__ int64_t scratch[32];
    __shared__ int page_first[kThreads], tok_first[kThreads], len_of[kThreads];
    __shared__ int n_served;
    let_next_start();
    wait_for_previous();
    const int tid = threadIdx.x;
    const int64_t free_n = min(max(static_cast<int64_t>(*free_count), int64_t(0)), free_cap);
    int64_t page_base = 0, tok_base = 0;               // of the block of requests
    int64_t taken = 0;
    for (int b0 = 0; b0 < B; b0 += kThreads) {
        const int b = b0 + tid, n_b = min(kThreads, B - b0);
        const int64_t len = b < B ? max(lens[b], 0) : 0;
        const int64_t add = b < B ? max(new_tokens[b], 0) : 0;
        const int64_t owned = (len + P - 1) / P;
        int64_t all_tok, all_pages;
        const int64_t tok_end = block_scan(add, scratch, all_tok) + tok_base;
        int64_t need = (len + add + P - 1) / P - owned;
        if (owned + need > ld || len + add > INT32_MAX || tok_end > n_slots) need = kNever;
        const int64_t page_end = block_scan(need, scratch, all_pages) + page_base;
        const bool served = page_end <= free_n;
        if (tid == 0) n_served = 0;
        page_first[tid] = static_cast<int>(min(page_end - need, int64_t(INT32_MAX)));
        tok_first[tid] = static_cast<int>(min(tok_end - add, int64_t(INT32_MAX)));
        len_of[tid] = served ? static_cast<int>(len) : -1;
        __syncthreads();
        if (b < B) {
            token_begin[b] = tok_first[tid];
            if (b == B - 1) token_begin[B] = static_cast<int>(min(tok_end, int64_t(INT32_MAX)));
            start[b] = len_of[tid];
            if (served) {
                lens[b] = static_cast<int>(len + add);
                atomicMax(&n_served, tid + 1);         // (the served ones come first: the sums ascend)
            }
        }
        __syncthreads();
        const int n_ok = n_served;
        const int64_t pages_end = n_ok > 0 ? (n_ok < n_b ? static_cast<int64_t>(page_first[n_ok]) : page_base + all_pages) : page_base;
        for (int64_t i = page_base + tid; i < pages_end; i += kThreads) {
            const int r = find_last(page_first, n_ok, static_cast<int>(i));
            const int64_t p = pages_of(len_of[r], P) + (i - page_first[r]);
            table[(b0 + r) * ld + p] = free_pages[free_n - 1 - i];
        }
        if (n_ok > 0) taken = pages_end;
        if (write_slots) {
            const int64_t t_end = min(tok_base + all_tok, n_slots);
            for (int64_t t = tok_base + tid; t < t_end; t += kThreads) {
                const int r = find_last(tok_first, n_b, static_cast<int>(t));
                int64_t slot = -1;
                if (len_of[r] >= 0) {
                    const unsigned pos = static_cast<unsigned>(len_of[r]) + static_cast<unsigned>(t - tok_first[r]);     // (below 2^31)
                    const unsigned p = pos / static_cast<unsigned>(P), had = pages_of(len_of[r], P);
                    const int page = p < had ? table[(b0 + r) * ld + p] : free_pages[free_n - 1 - (page_first[r] + static_cast<int>(p - had))];
                    if (page >= 0) slot = static_cast<int64_t>(page) * P + (pos - p * P);
                }
                slots[t] = slot;
                if (seq) seq[t] = b0 + r;
            }
        }
        page_base += all_pages;
        tok_base += all_tok;
        __syncthreads();
    }
    if (tid == 0) {
        *free_count = static_cast<int>(free_n - taken);
        if (B == 0) token_begin[0] = 0;
    }
    if (write_slots)
        for (int64_t t = min(tok_base, n_slots) + tid; t < n_slots; t += kThreads) {
            slots[t] = -1;
            if (seq) seq[t] = -1;
        }
}

__global__ void __launch_bounds__(256)
page_slots_kernel(const int32_t* table, int64_t ld, const int32_t* token_begin, const int32_t* start, int B, int P, int64_t* slots, int64_t n_slots,
                  int32_t* seq) {
    let_next_start();
    wait_for_previous();
    for (int64_t t = blockIdx.x * int64_t(256) + threadIdx.x; t < n_slots; t += gridDim.x * int64_t(256)) {
        int64_t slot = -1;
        int r = -1;
        if (t < token_begin[B]) {
            r = find_last(token_begin, B, static_cast<int32_t>(t));
            const int first = start[r];
            if (first >= 0) {
                const unsigned pos = static_cast<unsigned>(first) + static_cast<unsigned>(t - token_begin[r]);
                const unsigned p = pos / static_cast<unsigned>(P);
                const int page = table[r * ld + p];
                if (page >= 0) slot = static_cast<int64_t>(page) * P + (pos - p * P);
            }
        }
        slots[t] = slot;
        if (seq) seq[t] = r;
    }
}

__global__ void __launch_bounds__(kThreads)
page_release_kernel(int32_t* table, int64_t ld, int32_t* lens, const int32_t* keep_lens, int B, int P, int32_t* free_pages, int64_t free_cap,
                    int32_t* free_count) {
    __shared__ int64_t scratch[32];
    __shared__ int back_first[kThreads], from[kThreads];
    let_next_start();
    wait_for_previous();
    const int tid = threadIdx.x;
    const int64_t free_n = min(max(static_cast<int64_t>(*free_count), int64_t(0)), free_cap);
    int64_t given = 0;                                 // pages so far
    for (int b0 = (B - 1) / kThreads * kThreads; b0 >= 0; b0 -= kThreads) {
        const int b = b0 + tid, n_b = min(kThreads, B - b0);
        int64_t back = 0, all;                         // entries that request b gives back
        int first = 0;                                 // from this one on
        if (b < B) {
            const int64_t len = max(lens[b], 0), kept = min(len, static_cast<int64_t>(keep_lens ? max(keep_lens[b], 0) : 0));
            first = pages_of(static_cast<unsigned>(kept), P);
            back = max(min(static_cast<int64_t>(pages_of(static_cast<unsigned>(len), P)), ld) - first, int64_t(0));
            lens[b] = static_cast<int>(kept);
        }
        back_first[tid] = static_cast<int>(block_scan(back, scratch, all) - back);
        from[tid] = first;
        __syncthreads();
        // the entries end to end, U a thread and the last ones first: each page lies on the stack behind those of the entries after it
        auto give = [&](auto entries) {
            constexpr int U = decltype(entries)::value;
            for (int64_t top = all - 1; top >= 0; top -= kThreads * U) {
                const int64_t i0 = top - tid * U;
                int32_t* entry[U];
                int page[U], n = 0, r = i0 >= 0 ? find_last(back_first, n_b, static_cast<int>(i0)) : 0;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int i = static_cast<int>(i0) - u;
                    entry[u] = nullptr;
                    page[u] = -1;
                    if (i0 < u) continue;
                    while (u > 0 && i < back_first[r]) --r;
                    entry[u] = table + (b0 + r) * ld + from[r] + (i - back_first[r]);
                    page[u] = *entry[u];
                }
                bool pages = true;                     // every entry is one
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    pages = pages && (entry[u] == nullptr || page[u] >= 0);
                    if (entry[u] != nullptr) *entry[u] = -1;
                    n += page[u] >= 0;
                }
                int64_t place = tid * U, n_all = min(top + 1, int64_t(kThreads * U));
                if (!__syncthreads_and(pages)) place = block_scan(n, scratch, n_all) - n;
                place += free_n + given;
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (page[u] >= 0) {
                        if (place < free_cap) free_pages[place] = page[u];
                        ++place;
                    }
                given += n_all;
            }
        };
        if (all <= kThreads) give(std::integral_constant<int, 1>());
        else give(std::integral_constant<int, kGiveBack>());
        __syncthreads();
    }
    if (tid == 0) *free_count = static_cast<int>(min(free_n + given, free_cap));
}

// Positions -> cache rows. VEC positions a thread (their loads are independent).
template <int VEC>
__global__ void __launch_bounds__(256)
page_rows_kernel(const int32_t* table, int64_t ld, const int32_t* seq, int B, const int32_t* positions, int64_t n_rows, int k, int P,
                 int32_t* rows) {
    let_next_start();
    wait_for_previous();
    const int per_row = k / VEC;
    const int64_t n = n_rows * per_row;
    for (int64_t i = blockIdx.x * int64_t(256) + threadIdx.x; i < n; i += gridDim.x * int64_t(256)) {
        const int64_t row = i / per_row;
        const int64_t b = seq ? seq[row] : row;
        int pos[VEC], out[VEC];
        if (VEC == 4) {
            const int4 v = reinterpret_cast<const int4*>(positions)[i];
            pos[0] = v.x; pos[1 % VEC] = v.y; pos[2 % VEC] = v.z; pos[3 % VEC] = v.w;
        } else {
            pos[0] = positions[i];
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const int p = static_cast<int>(static_cast<unsigned>(pos[j]) / static_cast<unsigned>(P));
            const int page = pos[j] >= 0 && p < ld && b >= 0 && b < B ? table[b * ld + p] : -1;
            const int64_t at = static_cast<int64_t>(page) * P + (pos[j] - p * P);
            out[j] = page >= 0 && at <= INT32_MAX ? static_cast<int>(at) : -1;
        }
        if (VEC == 4) reinterpret_cast<int4*>(rows)[i] = make_int4(out[0], out[1 % VEC], out[2 % VEC], out[3 % VEC]);
        else rows[i] = out[0];
    }
}

}  // namespace

cudaError_t launch_page_tables(int32_t* table, int64_t ld, int32_t* lens, const int32_t* new_tokens, int B, int P, const int32_t* free_pages,
                               int64_t free_cap, int32_t* free_count, int32_t* token_begin, int32_t* start, int64_t* slots, int64_t n_slots,
                               int32_t* seq, cudaStream_t stream, int* launches) {
    const bool one = n_slots <= kFewTokens;
    cudaError_t e = launch_behind(page_tables_kernel, dim3(1), kThreads, 0, stream, table, ld, lens, new_tokens, B, P, free_pages, free_cap, free_count,
                                  token_begin, start, slots, n_slots, seq, one);
    *launches += 1;
    if (e != cudaSuccess || one) return e;
    const unsigned grid = static_cast<unsigned>(n_slots < 256 * 2048 ? (n_slots + 255) / 256 : 2048);
    *launches += 1;
    return launch_behind(page_slots_kernel, dim3(grid), 256, 0, stream, static_cast<const int32_t*>(table), ld, static_cast<const int32_t*>(token_begin),
                         static_cast<const int32_t*>(start), B, P, slots, n_slots, seq);
}

cudaError_t launch_page_release(int32_t* table, int64_t ld, int32_t* lens, const int32_t* keep_lens, int B, int P, int32_t* free_pages,
                                int64_t free_cap, int32_t* free_count, cudaStream_t stream) {
    return launch_behind(page_release_kernel, dim3(1), kThreads, 0, stream, table, ld, lens, keep_lens, B, P, free_pages, free_cap, free_count);
}

cudaError_t launch_page_rows(const int32_t* table, int64_t ld, const int32_t* seq, int B, const int32_t* positions, int64_t n_rows, int k, int P,
                             int32_t* rows, cudaStream_t stream) {
    const bool four = k % 4 == 0 && (reinterpret_cast<uintptr_t>(positions) | reinterpret_cast<uintptr_t>(rows)) % 16 == 0;
    const int64_t n = n_rows * (four ? k / 4 : k);
    const unsigned grid = static_cast<unsigned>(n < 256 * 4096 ? (n + 255) / 256 : 4096);
    return four ? launch_behind(page_rows_kernel<4>, dim3(grid), 256, 0, stream, table, ld, seq, B, positions, n_rows, k, P, rows)
                : launch_behind(page_rows_kernel<1>, dim3(grid), 256, 0, stream, table, ld, seq, B, positions, n_rows, k, P, rows);
}

}  // namespace idxc
