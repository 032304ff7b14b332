// Log probabilities of given tokens, with rank, entropy and the most probable tokens.
//
// With c = log2(e) / T, a reference r near the row's largest x c, and y_i = x_i c - r (one fma, so that r's own rounding shifts all y_i
// alike), Z = sum 2^y_i, S = sum 2^y_i y_i:
//   log p_i = ln2 (y_i - log2 Z),   entropy = ln2 (log2 Z - S / Z),   lse = max / T + ln2 (log2 Z - y of the maximum)
// Every thread has a reference of its own, its largest logit so far (one that lags behind by up to 2^24 made S of numbers up to 24 times as
// large, and the entropy of a peaked row off by 2e-6; the times are equal); the threads' sums are brought to the row's maximum at the end.
// The shift is half a unit in the last place of r: harmless below 2^20 (1/16), more than 2^y holds from 2^32 on.  So no reference starts or
// goes below -2^20 (what lies far below it adds nothing to a row whose maximum does not), and a row, or slice, whose maximum is 2^20 from
// zero or more is summed again from y_i = (x_i - max) c.
//
// One pass over the row: a thread takes 8 logits at a time (a "chunk"), leaves the chunk's maximum in LDS, and adds its terms.
// The most probable tokens then come from few chunks: of the threads' maxima the num_top-th largest is a value that at least
// num_top logits reach; only chunks whose maximum is above it (and the first ones that equal it: ties go to the lower token) are read
// again, and what they hold is ranked by counting.  Nothing is sorted, and no list depends on the order of arrival.
//
// A workgroup takes a row, or (up to 128 rows) a slice of one, which a second launch joins.
//
// Rounding: exponents, terms and a thread's sums are fp32 (up to 32 chunks one after another, each added as a tree), and so is the join.
// Bound: HBM.  1024 rows of 128256 bf16 logits with 5 alternatives 55.5 us (4.7 TB/s; without any 53), 500 fp32 rows with 20 50.7 (5.1),
// 2000 unaligned rows of 50257 45.5 (4.4).  64 fp32 rows of 128256 with 20 alternatives 16.3: slices 12 (a chain of loads, sums, threshold,
// second look) and the join 4.7; one workgroup a row 21.8, two slices 18.5, eight instead of four 18.1.  Two stripes of chunks ahead against four: 55.7 / 56.4
// and 45.9 / 48.7.  Four rows of 1024: 5.8, latency.
#include "logprobs_plan.h"
#include "spd_internal.h"

#include <type_traits>

namespace spd {
namespace {

using plan::kChunk;

constexpr float kFloor = -1000.f;   // y of a logit of -inf (2^-1000 = 0, and 0 * -1000 = 0)
constexpr float kFar = 1048576.f;   // from here on max c is rounded too far for a reference
constexpr float kMost = 3.402823466e38f;
constexpr float kLowest = -kFar;    // reference of a thread that has seen nothing above
constexpr int kMostRead = 128;      // chunks that are read again
constexpr int kJoinThreads = 256, kJoinKeys = 1024;

// Larger logits first, then the lower token: whole numbers in that order, all different.  NaN counts as -inf.
__device__ __forceinline__ unsigned value_key(float x)
{
    const unsigned u = __float_as_uint((x == x ? x : -INFINITY) + 0.f);  // (both zeros are one value)
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key_value(unsigned u)
{
    return __uint_as_float((u & 0x80000000u) ? (u & 0x7fffffffu) : ~u);
}

template <bool BF16> __device__ __forceinline__ float logit(const LogprobsParams& p, long long at)
{
    if (BF16)
        return __uint_as_float((unsigned)((const unsigned short*)p.logits)[at] << 16);
    return ((const float*)p.logits)[at];
}

// A chunk's 8 logits: of a whole one in 16-byte loads, else one by one (-inf where there is none).
template <bool BF16> struct Chunk {
    uint4 v[BF16 ? 1 : 2];
    __device__ __forceinline__ void load(const char* at)
    {
        v[0] = *(const uint4*)at;
        if (!BF16)
            v[BF16 ? 0 : 1] = *(const uint4*)(at + 16);
    }
    // of places chunk * 8 on from `from`, of which only first .. last are there: 8 loads at once
    __device__ __forceinline__ void load_some(const char* from, int place, int first, int last)
    {
        unsigned w[BF16 ? 4 : 8];
#pragma unroll
        for (int e = 0; e < kChunk; ++e) {
            const int at = min(max(place + e, first), last);
            const bool there = at == place + e;
            if (BF16) {
                const unsigned b = ((const unsigned short*)from)[at], u = there ? b : 0xff80u;
                w[e >> 1] = (e & 1) ? w[e >> 1] | u << 16 : u;
            } else {
                const unsigned u = ((const unsigned*)from)[at];
                w[BF16 ? 0 : e] = there ? u : 0xff800000u;
            }
        }
        v[0] = make_uint4(w[0], w[1], w[2], w[3]);
        if (!BF16)
            v[BF16 ? 0 : 1] = make_uint4(w[BF16 ? 0 : 4], w[BF16 ? 0 : 5], w[BF16 ? 0 : 6], w[BF16 ? 0 : 7]);
    }
    __device__ __forceinline__ void get(float (&x)[kChunk]) const
    {
        const unsigned w[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
        if (BF16) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        } else {
            const uint4 b = v[BF16 ? 0 : 1];
            const unsigned u[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[i] = __uint_as_float(w[i]);
                x[4 + i] = __uint_as_float(u[i]);
            }
        }
    }
};

// A number that at least k of a wavefront's keys, S a lane, reach, and no more than `most` where there is one; else the k-th largest.
template <int S> __device__ __forceinline__ unsigned threshold_key(const unsigned (&key)[S], int k, int most)
{
    // leading bits that all keys have
    const unsigned one = __builtin_amdgcn_readfirstlane(key[0]);
    unsigned differ = 0u;
#pragma unroll
    for (int s = 0; s < S; ++s)
        differ |= key[s] ^ one;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        differ |= __shfl_xor(differ, o);
    differ = __builtin_amdgcn_readfirstlane(differ);
    if (differ == 0u)
        return one;
    const int top_bit = 31 - __clz((int)differ);
    unsigned floor = one & ~((2u << top_bit) - 1u);
    for (int bit = top_bit; bit >= 0; --bit) {
        const unsigned cand = floor | (1u << bit);
        int count = 0;
#pragma unroll
        for (int s = 0; s < S; ++s)
            count += __popcll(__ballot(key[s] >= cand));
        if (count >= k) {
            floor = cand;
            if (count <= most)
                break;
        }
    }
    return floor;
}

// The k-th largest of n keys, of(i) each (LDS): it (exact: false), or a number that exactly k of them reach (exact: true).
template <class F> __device__ __forceinline__ unsigned kth_key(F of, int n, int k, bool& exact)
{
    const int lane = threadIdx.x & 63;
    unsigned floor = 0u;
    exact = false;
    for (int bit = 31; bit >= 0 && !exact; --bit) {
        const unsigned cand = floor | (1u << bit);
        int count = 0;
        for (int i = 0; i < n; i += 64)
            count += __popcll(__ballot(i + lane < n && of(i + lane) >= cand));
        if (count >= k) {
            floor = cand;
            exact = count == k;
        }
    }
    return floor;
}

__device__ __forceinline__ int lanes_below(unsigned long long mask)
{
    return __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0u));
}

// State of a slice: its largest logit, the reference and the sums; where the logit is far from zero, it is the reference.
struct State {
    float m, r, z, s;
};

// The sums on reference r, not below their own.
__device__ __forceinline__ void onto(State& a, float r)
{
    const float d = fmaxf(a.r - r, kFloor), f = __builtin_amdgcn_exp2f(d);
    a.s = f * __builtin_fmaf(a.z, d, a.s);
    a.z *= f;
    a.r = r;
}

__device__ __forceinline__ bool is_far(float m, float c) { return m > -INFINITY && m < INFINITY && !(fabsf(m * c) < kFar); }

// Exponent of x.
__device__ __forceinline__ float exponent(const State& a, float c, float x)
{
    return is_far(a.m, c) ? (x - a.m) * c : __builtin_fmaf(x, c, -a.r);
}

// How far a slice's reference lies above that of its row.
__device__ __forceinline__ float step_of(const State& b, const State& row, float c)
{
    if (!(b.m > -INFINITY))
        return kFloor;  // (nothing in it)
    if (is_far(row.m, c))
        return is_far(b.m, c) ? (b.m - row.m) * c : __builtin_fmaf(-row.m, c, b.r);
    return is_far(b.m, c) ? __builtin_fmaf(b.m, c, -row.r) : b.r - row.r;
}

// T, and log2(e) / T.
struct Scale {
    float t, c;
};

// What a row's sums say of a logit x.
__device__ __forceinline__ float log_p(const State& a, float log2_z, const Scale& by, float x)
{
    if (!(a.m > -INFINITY) || !(x > -INFINITY))
        return -INFINITY;
    const float y = exponent(a, by.c, x);
    if (!(y > -INFINITY))  // (too far below for base 2)
        return (x - a.m) / by.t;
    return (y - log2_z) * kLn2;
}

__device__ __forceinline__ void write_row(const LogprobsParams& p, long long row, const State& a, const Scale& by, bool known, float given, int above)
{
    const bool empty = !(a.m > -INFINITY);
    const float log2_z = __builtin_amdgcn_logf(a.z);
    if (p.logprobs)
        p.logprobs[row] = known ? log_p(a, log2_z, by, given) : -INFINITY;
    if (p.ranks)
        p.ranks[row] = known ? above + 1 : 0;
    if (p.entropy)
        p.entropy[row] = empty ? 0.f : kLn2 * (log2_z - a.s / a.z);
    if (p.lse)
        p.lse[row] = empty ? -INFINITY : a.m / by.t + kLn2 * (log2_z - exponent(a, by.c, a.m));
}

__device__ __forceinline__ void write_top(const LogprobsParams& p, long long row, int at, unsigned long long key, const State& a, float log2_z, const Scale& by)
{
    if (p.top_tokens)
        p.top_tokens[row * p.top + at] = (int)(0xffffffffu - (unsigned)key);
    if (p.top_logprobs)
        p.top_logprobs[row * p.top + at] = log_p(a, log2_z, by, key_value((unsigned)(key >> 32)));
}

__device__ __forceinline__ Scale scale_of(const LogprobsParams& p, long long row)
{
    const float given = p.temperature ? p.temperature[row] : 1.f, t = given > 0.f ? given : 1.f;
    return {t, fminf(kLog2e / t, kMost)};  // (0 times it is 0)
}

// THREADS, STRIPES: a workgroup takes up to STRIPES times THREADS chunks.  PARTS: slices of rows, joined by another launch.
template <bool BF16, int THREADS, int STRIPES, bool PARTS>
__global__ __launch_bounds__(THREADS) __attribute__((amdgpu_waves_per_eu(BF16 || STRIPES < 32 ? 8 : 4))) void logprobs_kernel(LogprobsParams p, int slice, int slices)
{
    constexpr int kWaves = THREADS / 64, kAhead = 2;
    constexpr int kHot = SPD_MAX_TOP_TOKENS + 8;  // threads up to which all of their chunks are looked through
    // (otherwise fewer than `top` threads lie above the threshold, and every wavefront adds up to `top` chunks that equal it)
    constexpr int kHits = kHot * STRIPES + kWaves * SPD_MAX_TOP_TOKENS;
    static_assert(THREADS * STRIPES <= 65536, "chunk numbers of 16 bits");
    using Max = typename std::conditional<BF16, unsigned short, unsigned>::type;  // a chunk's maximum, all of its bits
    __shared__ union {
        Max maxima[THREADS * STRIPES];
        unsigned long long found[kMostRead * kChunk];  // once the maxima are done with
    } big;
    __shared__ union {
        unsigned thread_keys[THREADS];
        unsigned short hits[kHits];  // once the threads' keys are
    } lists;
    __shared__ unsigned short read_again[kMostRead];
    __shared__ State states[kWaves];
    __shared__ int counts[kWaves], num_hot, num_hits, num_found, num_read;
    __shared__ unsigned short hot_threads[kHot];
    __shared__ unsigned threshold;
    auto& maxima = big.maxima;
    auto& found = big.found;
    auto& hits = lists.hits;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const long long row = PARTS ? blockIdx.x / slices : blockIdx.x;
    const int part = PARTS ? blockIdx.x % slices : 0;
    const int first = part * slice, len = min((int)p.vocab - first, slice);
    const long long base = row * p.stride + first;
    constexpr int kElt = BF16 ? 2 : 4;
    // chunks start on 16 bytes: `ahead` places of the first one lie in front of the slice
    const int ahead = (int)(((size_t)p.logits / kElt + (size_t)base) % (16 / kElt)), places = ahead + len;
    const int chunks = (places + kChunk - 1) / kChunk;
    const char* const from = (const char*)p.logits + (base - ahead) * kElt;
    const Scale by = scale_of(p, row);
    const float c = by.c;
    const int token = p.tokens ? p.tokens[row] : -1;
    const bool known = token >= 0 && token < (int)p.vocab;
    const float given = known ? fmaxf(logit<BF16>(p, row * p.stride + token), -INFINITY) : INFINITY;  // (a NaN counts as -inf)

    const auto whole = [&](int chunk) { return chunk * kChunk >= ahead && (chunk + 1) * kChunk <= places; };
    State a = {-INFINITY, kLowest, 0.f, 0.f};
    int above = 0;
    const auto take = [&](int chunk, const float (&x)[kChunk]) __attribute__((always_inline)) {
        float m = fmaxf(x[0], x[1]);
#pragma unroll
        for (int e = 2; e < kChunk; e += 2)
            m = fmaxf(m, fmaxf(x[e], x[e + 1]));
        if (p.top)
            maxima[chunk] = (Max)(__float_as_uint(m) >> (BF16 ? 16 : 0));
        a.m = fmaxf(a.m, m);
        if (__any(m > given)) {
#pragma unroll
            for (int e = 0; e < kChunk; ++e)
                above += __popcll(__ballot(x[e] > given));
        }
        const float r = fmaxf(m * c, kLowest);
        if (r > a.r)
            onto(a, r);
        float w[kChunk], s = 0.f;
#pragma unroll
        for (int e = 0; e < kChunk; ++e) {
            const float y = fmaxf(__builtin_fmaf(x[e], c, -a.r), kFloor);
            w[e] = __builtin_amdgcn_exp2f(y);
            s = __builtin_fmaf(w[e], y, s);
        }
        a.z += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
        a.s += s;
    };
    const int stripes = (chunks + THREADS - 1) / THREADS;
    for (int s0 = 0; s0 < stripes; s0 += kAhead) {
        Chunk<BF16> v[kAhead];
        const bool inside = s0 * THREADS * kChunk >= ahead && (s0 + kAhead) * THREADS * kChunk <= places;
        if (inside) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                v[i].load(from + (long long)((s0 + i) * THREADS + tid) * (kChunk * kElt));
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                float x[kChunk];
                v[i].get(x);
                take((s0 + i) * THREADS + tid, x);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int chunk = (s0 + i) * THREADS + tid;
                if (whole(chunk))
                    v[i].load(from + (long long)chunk * (kChunk * kElt));
                else
                    v[i].load_some(from, chunk * kChunk, ahead, places - 1);
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if ((s0 + i) * THREADS < chunks) {
                    float x[kChunk];
                    v[i].get(x);
                    take((s0 + i) * THREADS + tid, x);
                }
        }
    }

    // ---- sums over the workgroup, on the reference of the slice's maximum
    const unsigned own_key = tid < chunks ? value_key(a.m) : 0u;  // (a thread without a chunk of its own has no maximum)
    if (p.top)
        lists.thread_keys[tid] = own_key;
    float m = a.m;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        m = fmaxf(m, __shfl_xor(m, o));
    if (lane == 0) {
        states[wave].m = m;
        counts[wave] = above;
    }
    if (tid == 0)
        num_hot = num_hits = num_found = 0;
    __syncthreads();
    above = 0;
    for (int w = 0; w < kWaves; ++w) {
        m = fmaxf(m, states[w].m);
        above += counts[w];
    }
    if (is_far(m, c)) {
        a.z = a.s = 0.f;
        for (int chunk = tid; chunk < chunks; chunk += THREADS) {
            Chunk<BF16> v;
            v.load_some(from, chunk * kChunk, ahead, places - 1);
            float x[kChunk];
            v.get(x);
            for (int e = 0; e < kChunk; ++e) {
                const float y = fmaxf((x[e] - m) * c, kFloor), w = __builtin_amdgcn_exp2f(y);
                a.z += w;
                a.s = __builtin_fmaf(w, y, a.s);
            }
        }
        a.r = 0.f;
    } else {
        onto(a, fmaxf(m * c, kLowest));
    }
    a.m = m;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        a.z += __shfl_xor(a.z, o);
        a.s += __shfl_xor(a.s, o);
    }
    if (lane == 0) {
        states[wave].z = a.z;
        states[wave].s = a.s;
    }
    // ---- a value that at least `top` logits of the slice reach
    if (p.top && wave == 0) {
        unsigned key[kWaves];
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
            key[w] = lists.thread_keys[w * 64 + lane];
        const unsigned t = threshold_key(key, p.top, min(p.top + p.top / 2 + 2, kHot));
        if (lane == 0)
            threshold = t;
    }
    __syncthreads();
    a.z = a.s = 0.f;
    for (int w = 0; w < kWaves; ++w) {
        a.z += states[w].z;
        a.s += states[w].s;
    }
    LogprobsPart* const out_part = (LogprobsPart*)p.workspace + (PARTS ? blockIdx.x : 0);
    if (PARTS && tid == 0)
        *out_part = {a.m, a.r, a.z, a.s, above, 0};
    if (p.top == 0) {
        if (!PARTS && tid == 0)
            write_row(p, row, a, by, known, given, above);
        return;
    }

    // ---- chunks that reach the threshold.  Where few threads do, all of theirs that do; else (many that equal it) those above it and the
    // first ones of every wavefront that equal it.
    const auto key_of = [&](int chunk) { return value_key(__uint_as_float((unsigned)maxima[chunk] << (BF16 ? 16 : 0))); };
    const unsigned t = threshold;
    if (own_key >= t && own_key != 0u) {
        const int at = atomicAdd(&num_hot, 1);
        if (at < kHot)
            hot_threads[at] = (unsigned short)tid;
    }
    __syncthreads();
    if (num_hot <= kHot) {
        const int items = num_hot * stripes;
        for (int i = tid; i < items; i += THREADS) {
            const int chunk = i / num_hot * THREADS + hot_threads[i % num_hot];
            if (chunk < chunks && key_of(chunk) >= t)
                hits[atomicAdd(&num_hits, 1)] = (unsigned short)chunk;
        }
    } else {
        int ties = 0;
        for (int s = 0; s < stripes; ++s) {
            const int chunk = s * THREADS + tid;
            const unsigned key = chunk < chunks ? key_of(chunk) : 0u;
            const unsigned long long tied = __ballot(key == t && key != 0u);
            const bool tie = (tied >> lane & 1) && ties + lanes_below(tied) < p.top;
            ties += __popcll(tied);
            if (key > t || tie)
                hits[atomicAdd(&num_hits, 1)] = (unsigned short)chunk;
        }
    }
    __syncthreads();
    const int n = num_hits;
    if (n <= kMostRead) {
        if (tid < n)
            read_again[tid] = hits[tid];
        if (tid == 0)
            num_read = n;
    } else if (wave == 0) {
        // the same again among these: chunks above the top-th largest maximum, and of those that equal it the `top` lowest
        bool fits;
        const auto hit_key = [&](int i) { return key_of(hits[i]); };
        const unsigned t2 = kth_key(hit_key, n, p.top, fits);
        unsigned lowest = 0u;  // ~chunk from which on one that equals it is read
        if (!fits) {
            int equal = 0;
            for (int i = 0; i < n; i += 64)
                equal += __popcll(__ballot(i + lane < n && hit_key(i + lane) == t2));
            bool ignored;
            if (equal > p.top)
                lowest = kth_key([&](int i) { return hit_key(i) == t2 ? ~(unsigned)hits[i] : 0u; }, n, p.top, ignored);
        }
        int all = 0;
        for (int i = 0; i < n; i += 64) {
            const unsigned chunk = i + lane < n ? hits[i + lane] : 0u, key = key_of((int)chunk);
            const bool keep = i + lane < n && (fits ? key >= t2 : key > t2 || (key == t2 && ~chunk >= lowest));
            const unsigned long long kept = __ballot(keep);
            if (keep)
                read_again[all + lanes_below(kept)] = (unsigned short)chunk;
            all += __popcll(kept);
        }
        if (lane == 0)
            num_read = all;
    }
    __syncthreads();
    // ---- their logits, those that may be among the `top` largest, ranked by counting
    const int elements = num_read * kChunk;
    for (int i = tid; i < elements; i += THREADS) {
        const int at = (int)read_again[i / kChunk] * kChunk + i % kChunk;
        if (at >= ahead && at < places) {
            const float x = logit<BF16>(p, base - ahead + at);
            const unsigned key = value_key(x);
            if (key >= t)
                found[atomicAdd(&num_found, 1)] = (unsigned long long)key << 32 | (0xffffffffu - (unsigned)(first + at - ahead));
        }
    }
    __syncthreads();
    if (!PARTS && tid == THREADS - 1)  // (beside the first wavefronts' last work)
        write_row(p, row, a, by, known, given, above);
    const float log2_z = __builtin_amdgcn_logf(a.z);
    const int all = num_found;
    for (int i = tid; i < all; i += THREADS) {
        const unsigned long long key = found[i];
        int rank = 0;
        for (int q = 0; q < all; ++q)
            rank += found[q] > key;
        if (rank < p.top) {
            if (PARTS)
                ((unsigned long long*)((LogprobsPart*)p.workspace + p.rows * slices))[(long long)blockIdx.x * p.top + rank] = key;
            else
                write_top(p, row, rank, key, a, log2_z, by);
        }
    }
    if (PARTS && tid == 0)
        out_part->top = min(all, p.top);
}

// Joins a row's slices: sums on the reference of the row's maximum; the slices' sorted lists by their heads.
template <bool BF16> __global__ __launch_bounds__(kJoinThreads) void logprobs_join(LogprobsParams p, int slices)
{
    __shared__ unsigned long long listed[kJoinKeys];
    const long long row = blockIdx.x;
    const int lane = threadIdx.x & 63;  // (the sums are every wavefront's)
    const LogprobsPart* const parts = (const LogprobsPart*)p.workspace + row * slices;
    const unsigned long long* const keys = (const unsigned long long*)((const LogprobsPart*)p.workspace + p.rows * slices) + row * slices * p.top;
    const Scale by = scale_of(p, row);
    const float c = by.c;
    const int token = p.tokens ? p.tokens[row] : -1;
    const bool known = token >= 0 && token < (int)p.vocab;
    const float given = known ? fmaxf(logit<BF16>(p, row * p.stride + token), -INFINITY) : INFINITY;  // (a NaN counts as -inf)
    float m = -INFINITY;
    int above = 0;
    for (int i = lane; i < slices; i += 64) {
        m = fmaxf(m, parts[i].m);
        above += parts[i].above;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        m = fmaxf(m, __shfl_xor(m, o));
        above += __shfl_xor(above, o);
    }
    State a = {m, is_far(m, c) ? 0.f : fmaxf(m * c, kLowest), 0.f, 0.f};
    for (int i = lane; i < slices; i += 64) {
        State b = {parts[i].m, parts[i].r, parts[i].z, parts[i].s};
        b.r = step_of(b, a, c);
        onto(b, 0.f);
        a.z += b.z;
        a.s += b.s;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        a.z += __shfl_xor(a.z, o);
        a.s += __shfl_xor(a.s, o);
    }
    if (threadIdx.x == kJoinThreads - 1)  // (the first wavefronts have the lists)
        write_row(p, row, a, by, known, given, above);
    if (p.top == 0)
        return;
    const float log2_z = __builtin_amdgcn_logf(a.z);
    if (slices * p.top <= kJoinKeys) {
        // ranked by counting
        for (int i = threadIdx.x; i < slices * p.top; i += kJoinThreads)
            listed[i] = i % p.top < parts[i / p.top].top ? keys[i] : 0ull;
        __syncthreads();
        for (int i = threadIdx.x; i < slices * p.top; i += kJoinThreads) {
            const unsigned long long key = listed[i];
            int rank = 0;
            for (int q = 0; q < slices * p.top; ++q)
                rank += listed[q] > key;
            if (key != 0ull && rank < p.top)
                write_top(p, row, rank, key, a, log2_z, by);
        }
        return;
    }
    // the largest key below the last one, again and again: the first of every list that is
    unsigned long long last = ~0ull;
    for (int k = 0; k < p.top; ++k) {
        unsigned long long best = 0ull;
        for (int i = threadIdx.x; i < slices; i += kJoinThreads) {
            const int n = parts[i].top;
            for (int e = 0; e < n; ++e) {
                const unsigned long long key = keys[(long long)i * p.top + e];
                if (key < last) {
                    best = key > best ? key : best;
                    break;
                }
            }
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const unsigned long long other = __shfl_xor(best, o);
            best = other > best ? other : best;
        }
        __syncthreads();
        if (lane == 0)
            listed[threadIdx.x >> 6] = best;
        __syncthreads();
        for (int w = 0; w < kJoinThreads / 64; ++w)
            best = listed[w] > best ? listed[w] : best;
        last = best;
        if (threadIdx.x == 0)
            write_top(p, row, k, best, a, log2_z, by);
    }
}

template <bool BF16, int THREADS, int STRIPES> void run(const LogprobsParams& p, int slice, int slices, hipStream_t s)
{
    if (slices > 1)
        hipLaunchKernelGGL((logprobs_kernel<BF16, THREADS, STRIPES, true>), dim3((unsigned)(p.rows * slices)), dim3(THREADS), 0, s, p, slice, slices);
    else
        hipLaunchKernelGGL((logprobs_kernel<BF16, THREADS, STRIPES, false>), dim3((unsigned)p.rows), dim3(THREADS), 0, s, p, slice, slices);
}

template <bool BF16> hipError_t run_all(const LogprobsParams& p, hipStream_t s)
{
    const plan::LogprobsPlan pl = plan::make_logprobs_plan(p.rows, p.vocab);
    if (pl.threads == 256)
        pl.stripes == 4 ? run<BF16, 256, 4>(p, pl.slice, pl.slices, s) : run<BF16, 256, 8>(p, pl.slice, pl.slices, s);
    else if (pl.stripes == 8)
        run<BF16, 512, 8>(p, pl.slice, pl.slices, s);
    else if (pl.stripes == 16)
        run<BF16, 512, 16>(p, pl.slice, pl.slices, s);
    else
        run<BF16, 512, 32>(p, pl.slice, pl.slices, s);
    hipError_t rc = hipGetLastError();
    if (rc == hipSuccess && pl.slices > 1) {
        hipLaunchKernelGGL((logprobs_join<BF16>), dim3((unsigned)p.rows), dim3(kJoinThreads), 0, s, p, pl.slices);
        rc = hipGetLastError();
    }
    return rc;
}

}  // namespace

hipError_t launch_token_logprobs(const LogprobsParams& p, hipStream_t s)
{
    return p.bf16 ? run_all<true>(p, s) : run_all<false>(p, s);
}

}  // namespace spd
