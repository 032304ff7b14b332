// Which tokens of a cache stay (select_kv_tokens), and the copies that bring them together (compact_kv).
//
// Selection: the c-th largest weight of the tokens that are not kept by their place is found digit by digit (four digits
// of eight bits, a histogram each); of the tokens that equal it the lowest stay.  A workgroup a row.
//
// Compaction: source[i] >= i, so a workgroup that takes its places in ascending order, and reads every group of
// places before it writes them, overwrites nothing that it still has to read.
#include "spd_internal.h"

namespace spd {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// Weights as whole numbers in their order; NaN below all.
__device__ __forceinline__ unsigned key_of(float w)
{
    const unsigned u = __float_as_uint(w == 0.f ? 0.f : w);
    return w != w ? 0u : (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// Places before this thread's for which `yes` holds, and their number over the workgroup.
__device__ __forceinline__ int before(bool yes, int* lds, int& all)
{
    const unsigned long long mine = __ballot(yes);
    const int wave = threadIdx.x >> 6;
    int count = __builtin_amdgcn_mbcnt_hi((unsigned)(mine >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mine, 0u));
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        lds[wave] = __popcll(mine);
    __syncthreads();
    all = 0;
    for (int w = 0; w < kWaves; ++w) {
        count += w < wave ? lds[w] : 0;
        all += lds[w];
    }
    return count;
}

__global__ __launch_bounds__(kThreads) void select_kernel(SelectParams p)
{
    __shared__ int hist[256], lds[kWaves], found[2];
    const int b = blockIdx.x / p.heads, j = blockIdx.x % p.heads, tid = threadIdx.x;
    const int n = max(min(p.lens[b], p.max_len), 0), m = min(n, p.budgets ? max(min(p.budgets[b], p.max_new), 0) : p.max_new);
    const int r = min(p.recent, m), f = min(p.sinks, m - r), c = m - r - f;
    const float* const w = p.weights + (long long)blockIdx.x * p.stride;
    int* const source = p.source + (long long)blockIdx.x * p.source_stride;
    if (j == 0 && tid == 0)
        p.new_lens[b] = m;
    if (m == n) {
        for (int i = tid; i < m; i += kThreads)
            source[i] = i;
        return;
    }
    // the c-th largest of tokens f .. n - r - 1: key `floor`, `ties` of which stay
    unsigned floor = 0u, mask = 0u;
    int ties = c;
    for (int shift = 24; shift >= 0 && c > 0; shift -= 8) {
        hist[tid] = 0;
        __syncthreads();
        for (int t = f + tid; t < n - r; t += kThreads) {
            const unsigned key = key_of(w[t]);
            if ((key & mask) == floor)
                atomicAdd(&hist[key >> shift & 255u], 1);
        }
        __syncthreads();
        if (tid == 0) {
            int digit = 255, above = 0;
            while (above + hist[digit] < ties)
                above += hist[digit--];
            found[0] = digit;
            found[1] = above;
        }
        __syncthreads();
        floor |= (unsigned)found[0] << shift;
        mask |= 255u << shift;
        ties -= found[1];
    }
    // Places 0 .. m - r - 1 ("early"): tokens that stay, and gaps between them, which tokens m - r .. n - r - 1 that stay fill.  Both are
    // walked in ascending order, gaps and the tokens that fill them in step.
    __shared__ int gaps[kThreads];
    const int early = m - r;
    int tied = 0;  // ties in front of the walk
    const auto stays = [&](int t, int end) {
        const unsigned key = t < end ? key_of(w[t]) : 0u;
        const bool middle = t >= f && t < end && c > 0, tie = middle && key == floor;
        int all;
        const int rank = tied + before(tie, lds, all);
        tied += all;
        return (t < f && t < end) || (middle && key > floor) || (tie && rank < ties);
    };
    for (int t0 = 0; t0 < early; t0 += kThreads) {
        const int t = t0 + tid;
        const bool here = stays(t, early);
        if (t < early)
            source[t] = here ? t : -1;
    }
    __syncthreads();
    int listed = 0, used = 0, looked = 0;  // gaps in the list, those filled, and how far the places were looked through
    for (int t0 = early; t0 < n - r; t0 += kThreads) {
        const int t = t0 + tid;
        const bool here = stays(t, n - r);
        int moving, done = 0;
        const int nth = before(here, lds, moving);
        while (done < moving) {
            if (used == listed) {
                listed = used = 0;
                while (listed == 0 && looked < early) {
                    const bool gap = looked + tid < early && source[looked + tid] < 0;
                    const int at = before(gap, lds, listed);
                    if (gap)
                        gaps[at] = looked + tid;
                    looked += kThreads;
                }
                __syncthreads();
            }
            const int take = min(moving - done, listed - used);
            if (take <= 0)
                break;  // (there are as many gaps as tokens that fill them)
            if (here && nth >= done && nth < done + take)
                source[gaps[used + nth - done]] = t;
            __syncthreads();
            used += take;
            done += take;
        }
    }
    for (int i = early + tid; i < m; i += kThreads)
        source[i] = n - m + i;
}

__global__ __launch_bounds__(kThreads) void compact_kernel(CompactParams p)
{
    constexpr int kEach = 4;
    const int which = blockIdx.x & 1, j = (blockIdx.x >> 1) % p.Hkv, b = (blockIdx.x >> 1) / p.Hkv, tid = threadIdx.x;
    const int m = max(min(p.new_lens[b], p.max_new), 0);
    const int* const source = p.source + b * p.seq_stride + j * p.head_stride;
    const int in0 = p.indptr[b], out0 = p.out_indptr[b], per = p.page_size ? 16 : 1;
    const long long held = (long long)(p.indptr[b + 1] - in0) * per, room = (long long)(p.out_indptr[b + 1] - out0) * per;
    const uint4* const from = (const uint4*)(which ? p.v : p.k);
    uint4* const to = (uint4*)(which ? p.v_out : p.k_out);
    const auto at = [&](const int* pages, int first, int t) {
        return p.page_size ? (((long long)pages[first + (t >> 4)] * p.Hkv + j) * 16 + (t & 15)) * p.head_u4
                           : (long long)(first + t) * p.stride_u4 + (long long)j * p.head_u4;
    };
    // pieces of the places in order, kEach a thread at a time, all read before any is written
    const long long pieces = (long long)m * p.head_u4;
    for (long long i0 = 0; i0 < pieces; i0 += kEach * kThreads) {
        uint4 v[kEach];
        long long dst[kEach];
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const long long i = i0 + e * kThreads + tid;
            dst[e] = -1;
            v[e] = make_uint4(0u, 0u, 0u, 0u);
            if (i < pieces) {
                const int place = (int)(i / p.head_u4), piece = (int)(i % p.head_u4), src = source[place];
                if (src >= place && src < held && place < room && !(p.in_place && src == place)) {
                    v[e] = from[at(p.pages, in0, src) + piece];
                    dst[e] = at(p.out_pages, out0, place) + piece;
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kEach; ++e)
            if (dst[e] >= 0)
                to[dst[e]] = v[e];
    }
    if (which == 0 && p.weights) {
        const float* const w = p.weights + ((long long)b * p.Hkv + j) * p.weights_stride;
        float* const out = p.weights_out + ((long long)b * p.Hkv + j) * p.weights_stride;
        for (int i0 = 0; i0 < m; i0 += kThreads) {
            const int i = i0 + tid, src = i < m ? source[i] : -1;
            const float x = src >= i && src < p.weights_stride ? w[src] : 0.f;
            __syncthreads();
            if (i < m && src >= i)
                out[i] = x;
        }
        __syncthreads();
        for (long long i = m + tid; i < p.weights_stride; i += kThreads)
            out[i] = 0.f;
    }
    if (which == 0 && j == 0 && tid == 0 && p.lens_out)
        p.lens_out[b] = m;
}

}  // namespace

hipError_t launch_select_kv(const SelectParams& p, hipStream_t s)
{
    hipLaunchKernelGGL(select_kernel, dim3((unsigned)(p.seqs * p.heads)), dim3(kThreads), 0, s, p);
    return hipGetLastError();
}

hipError_t launch_compact_kv(const CompactParams& p, hipStream_t s)
{
    hipLaunchKernelGGL(compact_kernel, dim3((unsigned)(2 * p.B * p.Hkv)), dim3(kThreads), 0, s, p);
    return hipGetLastError();
}

}  // namespace spd
