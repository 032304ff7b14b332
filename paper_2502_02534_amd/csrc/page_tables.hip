// Page tables, slot map and granted lengths of requests from their lengths, on the device, so that a server's
// step needs no round trip to the host between admitting requests and running them.
//
// need_i = pages request i lacks; a request is served while the running sum of need fits the free list (and
// always when it needs nothing).  Three running sums follow: pages, free pages and new tokens.  One workgroup
// takes the sums, then every entry of the page list and of the slot map is found by bisection.
#include "spd_internal.h"

namespace spd {
namespace {

constexpr int kScanThreads = 1024;
constexpr int kThreads = 256;
constexpr int kPerThread = 4;  // entries of the page list or the slot map

// Inclusive sums over the workgroup, in place; `all` gets the total.  `lds` holds one value per wavefront.
template <int N, typename T>
__device__ __forceinline__ void block_sums(T (&x)[N], T (&all)[N], T* lds)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const T y = __shfl_up(x[k], o);
            x[k] += lane >= o ? y : (T)0;
        }
    __syncthreads();  // the last round's values have been read
    if (lane == 63)
#pragma unroll
        for (int k = 0; k < N; ++k)
            lds[k * (kScanThreads / 64) + wave] = x[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
        T before = 0, sum = 0;
        for (int w = 0; w < kScanThreads / 64; ++w) {
            const T y = lds[k * (kScanThreads / 64) + w];
            before += w < wave ? y : (T)0;
            sum += y;
        }
        x[k] += before;
        all[k] = sum;
    }
}

__global__ __launch_bounds__(kScanThreads) void page_sums_kernel(PageTableParams p)
{
    __shared__ long long lds64[kScanThreads / 64];
    __shared__ int lds32[3 * (kScanThreads / 64)];
    const int begin = p.free_begin ? *p.free_begin : 0;
    const long long room = p.num_free - begin;
    long long needed = 0;            // by all requests so far
    int pages = 0, taken = 0, fresh = 0;  // granted so far: pages, free pages, new tokens
    if (threadIdx.x == 0)
        p.page_indptr[0] = p.new_indptr[0] = 0;
    for (long long i0 = 0; i0 < p.n; i0 += kScanThreads) {
        const long long i = i0 + threadIdx.x;
        int held = 0, had = 0, want = 0;
        if (i < p.n) {
            if (p.held_lens) {
                had = p.held_lens[i];
                held = p.held_indptr[i + 1] - p.held_indptr[i];
            }
            want = max(p.lens[i], max(had, 0));
        }
        const long long pages_wanted = ((long long)want + p.page_size - 1) / p.page_size;
        const int need = (int)max(pages_wanted - held, 0ll);
        long long upto[1] = {need}, all[1];
        block_sums(upto, all, lds64);
        const bool granted = need == 0 || needed + upto[0] <= room;
        needed += all[0];
        const int get = granted ? need : 0, len = granted ? want : had;
        int sums[3] = {held + get, get, len - had}, totals[3];
        block_sums(sums, totals, lds32);
        if (i < p.n) {
            p.page_indptr[i + 1] = pages + sums[0];
            p.new_indptr[i + 1] = fresh + sums[2];
            p.lens_out[i] = len;
            p.first_free[i] = begin + taken + sums[1] - get;
        }
        pages += totals[0];
        taken += totals[1];
        fresh += totals[2];
    }
    if (threadIdx.x == 0)
        *p.free_end = begin + taken;
}

// The range of `indptr` that place t lies in: the last i with indptr[i] <= t.
__device__ __forceinline__ int range_of(const int* indptr, int n, long long t)
{
    int lo = 0, hi = n;  // indptr[lo] <= t < indptr[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (indptr[mid] <= t)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

__device__ __forceinline__ int page_of(const PageTableParams& p, int i, int k)
{
    const int first = p.held_lens ? p.held_indptr[i] : 0, held = p.held_lens ? p.held_indptr[i + 1] - first : 0;
    return k < held ? p.held_pages[first + k] : p.free_pages[p.first_free[i] + k - held];
}

__global__ __launch_bounds__(kThreads) void page_fill_kernel(PageTableParams p, unsigned page_blocks)
{
    const int n = (int)p.n;
    const bool slots = blockIdx.x >= page_blocks;
    const long long first = (long long)(blockIdx.x - (slots ? page_blocks : 0u)) * kThreads * kPerThread + threadIdx.x;
    const int* indptr = slots ? p.new_indptr : p.page_indptr;
    const long long total = indptr[n], most = slots ? p.max_tokens : p.max_pages;
#pragma unroll
    for (int u = 0; u < kPerThread; ++u) {
        const long long t = first + u * kThreads;
        if (t >= most)
            return;
        long long got = -1;
        if (t < total) {
            const int i = range_of(indptr, n, t);
            const int k = (int)(t - indptr[i]);
            if (slots) {
                const int at = (p.held_lens ? p.held_lens[i] : 0) + k;
                got = (long long)page_of(p, i, at / p.page_size) * p.page_size + at % p.page_size;
            } else {
                got = page_of(p, i, k);
            }
        }
        if (slots)
            p.slot_map[t] = got;
        else
            p.page_indices[t] = (int)got;
    }
}

}  // namespace

hipError_t launch_page_tables(const PageTableParams& p, hipStream_t s)
{
    hipLaunchKernelGGL(page_sums_kernel, dim3(1), dim3(kScanThreads), 0, s, p);
    const long long per_block = (long long)kThreads * kPerThread;
    const long long page_blocks = (p.max_pages + per_block - 1) / per_block;
    const long long slot_blocks = p.slot_map ? (p.max_tokens + per_block - 1) / per_block : 0;
    if (page_blocks + slot_blocks > 0)
        hipLaunchKernelGGL(page_fill_kernel, dim3((unsigned)(page_blocks + slot_blocks)), dim3(kThreads), 0, s, p, (unsigned)page_blocks);
    return hipGetLastError();
}

}  // namespace spd
