// Page tables, slot map and granted lengths of requests from their lengths, on the device, so that a server's
// step needs no round trip to the host between admitting requests and running them.
//
// need_i = pages request i lacks; a request is served while the running sum of need fits the free list (and
// always when it needs nothing).  Three running sums follow: pages, free pages and new tokens.  Every entry of the page
// list and of the slot map is then found by bisection in the sums.
//
// PACKED: the rows of new tokens were packed before anything was granted.  A fourth running sum counts the tokens asked for, the
// slot map follows it, and the places of refused requests get no slot.
//
// Up to kFew requests are one launch: every workgroup takes the sums of all requests by itself, into LDS, and fills
// its share of the entries (a second launch that waits for the first costs more than the sums).  More requests are
// two launches: one workgroup leaves the sums in memory, the others bisect there.
//
// Bound: latency.  8 requests of 1k to 16k tokens (77.5k slots) 4.7 us, 1024 requests that grow by up to 16 tokens each 6.4 (in two launches
// 10.5 and 17.5 us a call, now 5.9 and 6.1; 2048 requests 9.4 and, in two launches, 25.8).  5000 requests 34.8 us a call, 21 of them the one
// workgroup's sums.
#include "spd_internal.h"

#include <type_traits>

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
#pragma unroll 4
        for (int w = 0; w < kScanThreads / 64; ++w) {
            const T y = lds[k * (kScanThreads / 64) + w];
            before += w < wave ? y : (T)0;
            sum += y;
        }
        x[k] += before;
        all[k] = sum;
    }
}

// A count of tokens that is past 32 bits: no row of any tensor here has such a place.
__device__ __forceinline__ int most_int(long long x) { return (int)min(x, 0x7fffffffll); }

template <bool PACKED>
__global__ __launch_bounds__(kScanThreads) void page_sums_kernel(PageTableParams p)
{
    constexpr int kWide = PACKED ? 2 : 1;
    __shared__ long long lds64[kWide * (kScanThreads / 64)];
    __shared__ int lds32[3 * (kScanThreads / 64)];
    const int begin = p.free_begin ? *p.free_begin : 0;
    const long long room = p.num_free - begin;
    long long needed = 0, asked = 0;  // by all requests so far: pages, new tokens
    int pages = 0, taken = 0, fresh = 0;  // granted so far: pages, free pages, new tokens
    if (threadIdx.x == 0) {
        p.page_indptr[0] = p.new_indptr[0] = 0;
        if (PACKED)
            p.packed_indptr[0] = 0;
    }
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
        long long upto[kWide], all[kWide];
        upto[0] = need;
        if (PACKED)
            upto[kWide - 1] = (long long)want - had;
        block_sums(upto, all, lds64);
        const bool granted = need == 0 || needed + upto[0] <= room;
        needed += all[0];
        if (PACKED) {
            if (i < p.n) {
                p.packed_indptr[i + 1] = most_int(asked + upto[kWide - 1]);
                p.packed_lens[i] = granted ? want : 0;
            }
            asked += all[kWide - 1];
        }
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
    const bool packed = slots && p.packed_indptr;
    const int* indptr = packed ? p.packed_indptr : slots ? p.new_indptr : p.page_indptr;
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
            if (packed && p.new_indptr[i + 1] == p.new_indptr[i]) {  // refused
            } else if (slots) {
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

// ---- one launch ------------------------------------------------------------------------------------------------
constexpr int kFew = 2048;
constexpr int kFewThreads = 512;
constexpr int kEach = kFew / kFewThreads;  // requests a thread
constexpr int kFill = 2;                   // entries a thread

// Sums over the wavefronts before this one, of one value a wavefront in `lds`.
template <typename T, typename F> __device__ __forceinline__ T earlier(const T* lds, F add)
{
    T x = 0;
#pragma unroll
    for (int w = 0; w < kFewThreads / 64 - 1; ++w)
        x = add(x, w < (int)(threadIdx.x >> 6) ? lds[w] : (T)0);
    return x;
}

template <bool HELD, bool PACKED>
__global__ __launch_bounds__(kFewThreads) void page_tables_kernel(PageTableParams p, unsigned page_blocks)
{
    __shared__ int page_starts[kFew + 1], new_starts[kFew + 1], free_starts[kFew];
    __shared__ int held_first[HELD ? kFew + 1 : 1], had_tokens[HELD ? kFew : 1], packed_starts[PACKED ? kFew + 1 : 1];
    __shared__ uint32_t wave_need[kFewThreads / 64], wave_asked[PACKED ? kFewThreads / 64 : 1];
    __shared__ int wave_pages[kFewThreads / 64], wave_taken[kFewThreads / 64], wave_fresh[kFewThreads / 64];
    const int n = (int)p.n, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int begin = p.free_begin ? *p.free_begin : 0;
    const uint32_t room = (uint32_t)max(p.num_free - begin, 0ll);
    const auto sat = [](uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); };
    const auto add = [](int a, int b) { return a + b; };
    int held[kEach], had[kEach], want[kEach];
    uint32_t need[kEach], mine = 0u, asked[kEach], my_asked = 0u;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int i = tid * kEach + k;
        held[k] = had[k] = want[k] = 0;
        if (i < n) {
            if constexpr (HELD) {
                const int first = p.held_indptr[i];
                held_first[i] = first;
                held[k] = p.held_indptr[i + 1] - first;
                had[k] = p.held_lens[i];
                had_tokens[i] = had[k];
                if (i == n - 1)
                    held_first[n] = first + held[k];
            }
            want[k] = max(p.lens[i], max(had[k], 0));
        }
        const unsigned pages = ((unsigned)want[k] + (unsigned)p.page_size - 1u) / (unsigned)p.page_size;
        need[k] = (uint32_t)max((int)pages - held[k], 0);
        mine = sat(mine, need[k]);
        if constexpr (PACKED) {
            asked[k] = my_asked;
            my_asked = sat(my_asked, (uint32_t)want[k] - (uint32_t)had[k]);
        }
    }
    uint32_t upto = mine;  // saturating: a sum past 2^32 fits no free list either
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t x = (uint32_t)__shfl_up((int)upto, o);
        upto = lane >= o ? sat(upto, x) : upto;
    }
    uint32_t before = (uint32_t)__shfl_up((int)upto, 1);
    before = lane == 0 ? 0u : before;
    if (lane == 63)
        wave_need[wave] = upto;
    uint32_t up_asked = my_asked;
    if constexpr (PACKED) {
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t x = (uint32_t)__shfl_up((int)up_asked, o);
            up_asked = lane >= o ? sat(up_asked, x) : up_asked;
        }
        if (lane == 63)
            wave_asked[wave] = up_asked;
        up_asked = (uint32_t)__shfl_up((int)up_asked, 1);
        up_asked = lane == 0 ? 0u : up_asked;  // of the lanes before
    }
    __syncthreads();
    before = sat(before, earlier(wave_need, sat));
    if constexpr (PACKED)
        up_asked = sat(up_asked, earlier(wave_asked, sat));
    int pages[kEach], taken[kEach], fresh[kEach];  // running sums within the thread
    int sum_pages = 0, sum_taken = 0, sum_fresh = 0;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        before = sat(before, need[k]);
        const bool granted = need[k] == 0u || before <= room;
        const int get = granted ? (int)need[k] : 0;
        if constexpr (PACKED) {
            const int i = tid * kEach + k;
            if (blockIdx.x == 0 && i < n)
                p.packed_lens[i] = granted ? want[k] : 0;
        }
        want[k] = granted ? want[k] : had[k];
        pages[k] = sum_pages;
        taken[k] = sum_taken;
        fresh[k] = sum_fresh;
        sum_pages += held[k] + get;
        sum_taken += get;
        sum_fresh += want[k] - had[k];
    }
    int up_pages = sum_pages, up_taken = sum_taken, up_fresh = sum_fresh;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int a = __shfl_up(up_pages, o), b = __shfl_up(up_taken, o), c = __shfl_up(up_fresh, o);
        up_pages += lane >= o ? a : 0;
        up_taken += lane >= o ? b : 0;
        up_fresh += lane >= o ? c : 0;
    }
    if (lane == 63) {
        wave_pages[wave] = up_pages;
        wave_taken[wave] = up_taken;
        wave_fresh[wave] = up_fresh;
    }
    __syncthreads();
    const int base_pages = up_pages - sum_pages + earlier(wave_pages, add);
    const int base_taken = begin + up_taken - sum_taken + earlier(wave_taken, add);
    const int base_fresh = up_fresh - sum_fresh + earlier(wave_fresh, add);
    const bool writes = blockIdx.x == 0;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int i = tid * kEach + k;
        if (i <= n) {  // (request n holds nothing: its starts are the totals)
            page_starts[i] = base_pages + pages[k];
            new_starts[i] = base_fresh + fresh[k];
            if (writes) {
                p.page_indptr[i] = base_pages + pages[k];
                p.new_indptr[i] = base_fresh + fresh[k];
            }
            if constexpr (PACKED) {
                packed_starts[i] = most_int(sat(up_asked, asked[k]));
                if (writes)
                    p.packed_indptr[i] = packed_starts[i];
            }
        }
        if (i < n) {
            free_starts[i] = base_taken + taken[k];
            if (writes)
                p.lens_out[i] = want[k];
        }
    }
    if (tid == kFewThreads - 1) {
        const int all = base_taken + sum_taken;
        if (n == kFew) {
            page_starts[n] = base_pages + sum_pages;
            new_starts[n] = base_fresh + sum_fresh;
            if (writes) {
                p.page_indptr[n] = base_pages + sum_pages;
                p.new_indptr[n] = base_fresh + sum_fresh;
            }
            if constexpr (PACKED) {
                packed_starts[n] = most_int(sat(up_asked, my_asked));
                if (writes)
                    p.packed_indptr[n] = packed_starts[n];
            }
        }
        if (writes)
            *p.free_end = all;
    }
    __syncthreads();
    const auto page_at = [&](int i, int k) -> int {
        const int first = HELD ? held_first[i] : 0, mine_held = HELD ? held_first[i + 1] - first : 0;
        return HELD && k < mine_held ? p.held_pages[first + k] : p.free_pages[free_starts[i] + k - mine_held];
    };
    const bool slots = blockIdx.x >= page_blocks;
    const long long first = (long long)(blockIdx.x - (slots ? page_blocks : 0u)) * kFewThreads * kFill + tid;
    const int* starts = slots ? PACKED ? packed_starts : new_starts : page_starts;
    const long long total = starts[n], most = slots ? p.max_tokens : p.max_pages;
#pragma unroll
    for (int u = 0; u < kFill; ++u) {
        const long long t = first + u * kFewThreads;
        if (t >= most)
            return;
        long long got = -1;
        if (t < total) {
            const int i = range_of(starts, n, t), k = (int)(t - starts[i]);
            if (PACKED && slots && new_starts[i + 1] == new_starts[i]) {  // refused
            } else if (slots) {
                const unsigned at = (unsigned)((HELD ? had_tokens[i] : 0) + k), page = at / (unsigned)p.page_size;
                got = (long long)page_at(i, (int)page) * p.page_size + (at - page * (unsigned)p.page_size);
            } else {
                got = page_at(i, k);
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
    if (p.n <= kFew) {
        const long long per_block = (long long)kFewThreads * kFill;
        const long long page_blocks = (p.max_pages + per_block - 1) / per_block;
        const long long slot_blocks = p.slot_map ? (p.max_tokens + per_block - 1) / per_block : 0;
        const long long blocks = page_blocks + slot_blocks > 0 ? page_blocks + slot_blocks : 1;
        const dim3 grid((unsigned)blocks), block(kFewThreads);
        // (with no page entries at all the one workgroup there is fills none)
        const unsigned first_slots = (unsigned)(slot_blocks > 0 ? page_blocks : blocks);
        const auto go = [&](auto held, auto packed) {
            hipLaunchKernelGGL((page_tables_kernel<decltype(held)::value, decltype(packed)::value>), grid, block, 0, s, p, first_slots);
        };
        const std::true_type yes{};
        const std::false_type no{};
        if (p.packed_indptr)
            p.held_lens ? go(yes, yes) : go(no, yes);
        else
            p.held_lens ? go(yes, no) : go(no, no);
        return hipGetLastError();
    }
    if (p.packed_indptr)
        hipLaunchKernelGGL(page_sums_kernel<true>, dim3(1), dim3(kScanThreads), 0, s, p);
    else
        hipLaunchKernelGGL(page_sums_kernel<false>, dim3(1), dim3(kScanThreads), 0, s, p);
    const long long per_block = (long long)kThreads * kPerThread;
    const long long page_blocks = (p.max_pages + per_block - 1) / per_block;
    const long long slot_blocks = p.slot_map ? (p.max_tokens + per_block - 1) / per_block : 0;
    if (page_blocks + slot_blocks > 0)
        hipLaunchKernelGGL(page_fill_kernel, dim3((unsigned)(page_blocks + slot_blocks)), dim3(kThreads), 0, s, p, (unsigned)page_blocks);
    return hipGetLastError();
}

}  // namespace spd
