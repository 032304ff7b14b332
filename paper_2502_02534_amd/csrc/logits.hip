// What stands between the logits and the sampler: which tokens a prompt holds (a bit per token of the vocabulary),
// and the logits shaped by penalties, biases and a grammar mask.
#include "spd_internal.h"

#include <float.h>
#include <type_traits>

namespace spd {
namespace {

// ---- which tokens occur in a prompt ----------------------------------------------------------------------
// One workgroup per prompt and stretch of the vocabulary: the stretch's bits are collected in LDS.  Bound: latency (the
// launch, one round trip for the prompt's range, one for kBatch tokens a thread at a time): one prompt of 8192 tokens 2.8 us, eight
// of 1024 to 16384 over 128256 ids 4.2.
constexpr int kMarkThreads = 1024;
constexpr int kMarkWords = 4096;  // of a stretch (131072 tokens)
constexpr int kBatch = 8;

__global__ __launch_bounds__(kMarkThreads) void mark_tokens_kernel(const int* tokens, const int* indptr, long long vocab,
                                                                   uint32_t* bits, long long stride, int accumulate)
{
    __shared__ uint32_t lds[kMarkWords];
    // (unsigned: past the last of up to 2^31 tokens a thread's place still fits)
    const unsigned first = (unsigned)max(indptr[blockIdx.x], 0), end = (unsigned)max(indptr[blockIdx.x + 1], 0);
    const long long all_words = (vocab + 31) / 32, word0 = (long long)blockIdx.y * kMarkWords;
    const int words = (int)min(all_words - word0, (long long)kMarkWords);
    uint32_t* row = bits + (long long)blockIdx.x * stride + word0;
    for (int w = threadIdx.x; w < words; w += kMarkThreads)
        lds[w] = accumulate ? row[w] : 0u;
    const int lo = (int)word0 * 32, len = (int)min(vocab - lo, (long long)words * 32);
    int id[kBatch];
    auto request = [&](unsigned t0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
            id[u] = tokens[min(t0 + threadIdx.x + u * kMarkThreads, end - 1)];
    };
    if (first < end)
        request(first);
    __syncthreads();
    for (unsigned t0 = first; t0 < end; t0 += kBatch * kMarkThreads) {
        if (t0 > first)
            request(t0);
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const unsigned at = (unsigned)id[u] - (unsigned)lo;
            if (t0 + threadIdx.x + u * kMarkThreads < end && id[u] >= 0 && at < (unsigned)len)
                atomicOr(&lds[at >> 5], 1u << (at & 31));
        }
    }
    __syncthreads();
    for (int w = threadIdx.x; w < words; w += kMarkThreads)
        row[w] = lds[w];
}

// ---- penalties, biases, grammar mask -----------------------------------------------------------------------
// One workgroup per row and slice of the vocabulary.  The tokens of the slice that occur in the row's history or biases
// ("listed", few) get a bit each and, by the number of bits before it, a place in a table of counts and biases; the logits
// then pass through once, four a thread, and only those whose bit is set look into the table.  A slice with more
// listed tokens than the table holds is taken in stretches as long as the table.  A wavefront has the logits of its
// tokens on their way before the table is begun, and takes a word of every bit row per lane, handed round with shuffles.
//
// Bound: HBM, logits read and written once.  1024 rows of 128256 bf16 logits, histories up to 2048 by steps, 8 prompts' bits, 16 biases and
// a grammar row each: 176 us, 4.5 TB/s (a cast of the same logits to fp32 136; histories row by row 165, none 151); 64 fp32 rows
// 18.1 us, 3.6 TB/s: reading the history, then the table, is a chain that the first slices wait for.  57 to 63 registers: four
// workgroups a CU (with 108, two: 198 us); 77, three, with eight rounds of fp32.
constexpr int kThreads = 512;
constexpr int kTable = 2048;         // places
constexpr int kEntries = 4;          // of the history, a thread: a history of kEntries * kThreads is read once
constexpr int kMaxSlice = 16384;     // tokens: a bit each
constexpr int kWords = kMaxSlice / 32;
static_assert(kWords <= kThreads, "one word a thread");
// Tokens of a slice with ROUNDS rounds of four tokens a lane.
constexpr int slice_tokens(int rounds) { return rounds * 4 * kThreads; }

// Four logits as they lie in memory, from a place that is aligned to its element only (the hardware takes any).
template <bool BF16> struct Four {
    uint32_t w[BF16 ? 2 : 4];
    __device__ __forceinline__ void load(const char* at, int m)  // m of them: up to four
    {
        typedef uint32_t __attribute__((ext_vector_type(2), aligned(2))) any2;
        typedef uint32_t __attribute__((ext_vector_type(4), aligned(4))) any4;
        if (m == 4) {
            if constexpr (BF16) {
                const any2 v = *reinterpret_cast<const any2*>(at);
                w[0] = v[0];
                w[1] = v[1];
            } else {
                const any4 v = *reinterpret_cast<const any4*>(at);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    w[i] = v[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < (BF16 ? 2 : 4); ++i)
                w[i] = 0u;
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (e < m) {
                    if constexpr (BF16)
                        w[e >> 1] |= (uint32_t)((const uint16_t*)at)[e] << (16 * (e & 1));
                    else
                        w[e] = ((const uint32_t*)at)[e];
                }
        }
    }
    __device__ __forceinline__ float get(int e) const
    {
        if constexpr (BF16)
            return __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
        else
            return __uint_as_float(w[e]);
    }
};

template <bool BF16, int ROUNDS>
__global__ __launch_bounds__(kThreads) void penalize_kernel(LogitsParams p, int slices)
{
    constexpr int slice_len = slice_tokens(ROUNDS), kTile = 256 * ROUNDS;
    static_assert(slice_len <= kMaxSlice, "a bit for every token");
    __shared__ uint32_t listed[kWords];
    __shared__ uint16_t before[kWords];  // listed tokens in the words before
    __shared__ uint32_t counts[kTable];
    __shared__ float bias[kTable];
    __shared__ int wave_sums[kThreads / 64];
    const int tid = threadIdx.x;
    // the rows of an XCD follow one another: they read the same lines of a step-major history and the same prompts' bits
    const unsigned unit = blockIdx.x >> 3, rows8 = (unsigned)((p.rows + 7) / 8);
    const long long r = (unsigned)__builtin_amdgcn_readfirstlane((blockIdx.x & 7) * rows8 + unit / (unsigned)slices);
    if (r >= p.rows)
        return;
    const int lo = __builtin_amdgcn_readfirstlane((int)(unit % (unsigned)slices)) * slice_len, hi = min((int)p.vocab, lo + slice_len);

    // x / rep as x * (inv + rest), the reciprocal in two floats: rounded once, in five instructions with the product for x <= 0, where
    // the division alone takes ten (1024 rows 190 us).  Exact so far as x * rest is, from |x| = 2^-110 on, and reciprocals are not subnormal.
    const float rep = p.repetition ? p.repetition[r] : 1.f;
    const bool repeats = rep != 1.f, usual_rep = rep >= 0x1p-60f && rep <= 0x1p60f;
    const auto uniform = [](float x) { return __uint_as_float((uint32_t)__builtin_amdgcn_readfirstlane((int)__float_as_uint(x))); };
    const float inv = uniform(1.f / rep), rest = uniform(fmaf(-rep, inv, 1.f) * inv);
    const float freq = p.frequency ? p.frequency[r] : 0.f, pres = p.presence ? p.presence[r] : 0.f;
    const long long prompt = !p.prompt_bits || !repeats ? -1 : p.prompt_of_row ? p.prompt_of_row[r] : r;
    const long long grammar = !p.allowed_bits ? -1 : p.allowed_of_row ? p.allowed_of_row[r] : r;
    const uint32_t* seen_bits = p.prompt_bits + (prompt < 0 ? 0 : prompt) * p.prompt_stride;
    const uint32_t* allowed_bits = p.allowed_bits + (grammar < 0 ? 0 : grammar) * p.allowed_stride;
    const int n = p.tokens ? min(p.token_lens[r], p.max_tokens) : 0;
    const int* mine = p.tokens + r * p.token_row_stride;
    const int b0 = p.bias_tokens ? p.bias_indptr[r] : 0, b1 = p.bias_tokens ? p.bias_indptr[r + 1] : 0;
    const char* in = (const char*)p.logits + r * p.stride * (BF16 ? 2 : 4);
    float* out = p.out + r * p.out_stride;

    const bool any = n > 0 || b1 > b0;
    int ids[kEntries];
    auto read_history = [&](int q0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kEntries; ++u) {
            const int q = q0 + tid + u * kThreads;
            const int id = mine[min(q, n - 1) * p.token_step_stride];
            ids[u] = q < n ? id : -1;
        }
    };
    if (n > 0)
        read_history(0);
    int step = slice_len;
    for (int s0 = lo; s0 < hi;) {
        // (opaque, here and in the rounds below, so that no place's address is worked out ahead and kept in registers)
        int me = tid;
        asm volatile("" : "+v"(me));
        const int len = min(step, hi - s0), words = (len + 31) / 32;
        // k = place in the stretch.  The wavefront's tile and the words of its bits, all at once
        const int lane = me & 63, tile0 = (me >> 6) * kTile, tile_len = min(len - tile0, kTile);
        Four<BF16> raw[ROUNDS];
        uint32_t seen_words = 0u, allowed_words = 0xffffffffu;
        const char* const from = in + (long long)(s0 + tile0) * (BF16 ? 2 : 4);
        if (tile_len == kTile) {
#pragma unroll
            for (int u = 0; u < ROUNDS; ++u)
                raw[u].load(from + (256 * u + 4 * lane) * (BF16 ? 2 : 4), 4);
        } else {
#pragma unroll
            for (int u = 0; u < ROUNDS; ++u)
                if (256 * u + 4 * lane < tile_len)
                    raw[u].load(from + (256 * u + 4 * lane) * (BF16 ? 2 : 4), min(4, tile_len - (256 * u + 4 * lane)));
        }
        if (32 * lane < tile_len) {
            const int w = (s0 + tile0) / 32 + lane;
            if (prompt >= 0)
                seen_words = seen_bits[w];
            if (grammar >= 0)
                allowed_words = allowed_bits[w];
        }
        if (any) {
            // every history entry of this stretch, and every bias entry
            auto each_token = [&](auto f) __attribute__((always_inline)) {
                for (int q0 = 0; q0 < n; q0 += kEntries * kThreads) {
                    if (n > kEntries * kThreads)
                        read_history(q0);
#pragma unroll
                    for (int u = 0; u < kEntries; ++u) {
                        const unsigned id = (unsigned)ids[u] - (unsigned)s0;  // (a negative token's is past any length)
                        if (ids[u] >= 0 && id < (unsigned)len)
                            f((int)id);
                    }
                }
            };
            auto each_bias = [&](auto f) __attribute__((always_inline)) {
                for (int k = b0 + me; k < b1; k += kThreads) {
                    const int token = p.bias_tokens[k];
                    const unsigned id = (unsigned)token - (unsigned)s0;
                    if (token >= 0 && id < (unsigned)len)
                        f((int)id, k);
                }
            };
            auto place = [&](int id) __attribute__((always_inline)) -> int {
                return before[id >> 5] + __popc(listed[id >> 5] & ((1u << (id & 31)) - 1u));
            };
            __syncthreads();  // the stretch before has been read
            if (me < words)
                listed[me] = 0u;
            for (int i = me; i < kTable; i += kThreads) {
                counts[i] = 0u;
                bias[i] = 0.f;
            }
            __syncthreads();
            each_token([&](int id) __attribute__((always_inline)) { atomicOr(&listed[id >> 5], 1u << (id & 31)); });
            each_bias([&](int id, int) __attribute__((always_inline)) { atomicOr(&listed[id >> 5], 1u << (id & 31)); });
            __syncthreads();
            const int bits = me < words ? __popc(listed[me]) : 0;
            int upto = bits;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int x = __shfl_up(upto, o);
                upto += (me & 63) >= o ? x : 0;
            }
            if ((me & 63) == 63)
                wave_sums[me >> 6] = upto;
            __syncthreads();
            int first = upto - bits, total = 0;
#pragma unroll
            for (int w = 0; w < kThreads / 64; ++w) {
                first += w < (me >> 6) ? wave_sums[w] : 0;
                total += wave_sums[w];
            }
            if (total > kTable) {  // (for everybody alike)
                step = kTable;
                continue;
            }
            if (me < words)
                before[me] = (uint16_t)first;
            __syncthreads();
            each_token([&](int id) __attribute__((always_inline)) { atomicAdd(&counts[place(id)], 1u); });
            each_bias([&](int id, int k) __attribute__((always_inline)) { bias[place(id)] = p.bias_values[k]; });
            __syncthreads();
        }
        auto repeated = [&](auto by_product, float x) __attribute__((always_inline)) -> float {
            if constexpr (decltype(by_product)::value)
                return fmaf(x, x > 0.f ? inv : rep, __builtin_amdgcn_fmed3f(x, 0.f, FLT_MAX) * rest);  // (an infinite x stays one)
            return x > 0.f ? x / rep : x * rep;
        };
        // one that is listed: its count and bias
        auto shape = [&](auto by_product, float x, bool seen, int k) __attribute__((always_inline)) -> float {
            const int at = before[k >> 5] + __popc(listed[k >> 5] & ((1u << (k & 31)) - 1u));
            const uint32_t c = counts[at];
            if (c != 0u && !seen && repeats)
                x = repeated(by_product, x);
            if (c != 0u)
                x = x - freq * (float)c - pres;
            return x + bias[at];
        };
        uint32_t listed_words = any && 32 * lane < tile_len ? listed[tile0 / 32 + lane] : 0u;
        float* const to = out + s0 + tile0;
        auto round = [&](int u, const Four<BF16>& four, auto full, auto by_product) __attribute__((always_inline)) {
            int at_lane = lane;
            asm volatile("" : "+v"(at_lane), "+v"(listed_words), "+v"(seen_words), "+v"(allowed_words));
            // the lane's four bits: of word 8 u + lane / 8, from bit 4 (lane % 8) on
            const int from_lane = 8 * u + (at_lane >> 3), shift = 4 * (at_lane & 7), k = 256 * u + 4 * at_lane;
            const uint32_t bits = any ? (uint32_t)__shfl((int)listed_words, from_lane) >> shift & 0xfu : 0u;
            const uint32_t seen = prompt >= 0 ? (uint32_t)__shfl((int)seen_words, from_lane) >> shift & 0xfu : 0u;
            const uint32_t allowed = grammar >= 0 ? (uint32_t)__shfl((int)allowed_words, from_lane) >> shift & 0xfu : 0xfu;
            if (full || k < tile_len) {
                float x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    x[e] = four.get(e);
                if (seen != 0u)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float y = repeated(by_product, x[e]);
                        x[e] = (seen >> e) & 1u ? y : x[e];
                    }
                if (bits != 0u)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if ((bits >> e) & 1u)
                            x[e] = shape(by_product, x[e], (seen >> e) & 1u, tile0 + k + e);
                if (allowed != 0xfu)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        x[e] = (allowed >> e) & 1u ? x[e] : -INFINITY;
                if (full || tile_len - k >= 4) {
                    typedef float __attribute__((ext_vector_type(4), aligned(4))) any4;
                    const any4 y = {x[0], x[1], x[2], x[3]};
                    *reinterpret_cast<any4*>(to + k) = y;
                } else {
#pragma unroll
                    for (int e = 0; e < 3; ++e)
                        if (e < tile_len - k)
                            to[k + e] = x[e];
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        if (!usual_rep) {  // (rare: its logits are read again, so that this copy of the code is short)
#pragma unroll 1
            for (int u = 0; u < ROUNDS; ++u) {
                const int k = 256 * u + 4 * lane;
                Four<BF16> four = {};
                if (k < tile_len)
                    four.load(from + k * (BF16 ? 2 : 4), min(4, tile_len - k));
                round(u, four, std::false_type{}, std::false_type{});
            }
        } else if (tile_len == kTile) {
#pragma unroll
            for (int u = 0; u < ROUNDS; ++u)
                round(u, raw[u], std::true_type{}, std::true_type{});
        } else {
#pragma unroll
            for (int u = 0; u < ROUNDS; ++u)
                round(u, raw[u], std::false_type{}, std::true_type{});
        }
        s0 += len;
    }
}

}  // namespace

hipError_t launch_mark_tokens(const int* tokens, const int* indptr, long long prompts, long long vocab, uint32_t* bits,
                              long long stride, bool accumulate, hipStream_t s)
{
    const long long words = (vocab + 31) / 32;
    hipLaunchKernelGGL(mark_tokens_kernel, dim3((unsigned)prompts, (unsigned)((words + kMarkWords - 1) / kMarkWords)), dim3(kMarkThreads),
                       0, s, tokens, indptr, vocab, bits, stride, accumulate ? 1 : 0);
    return hipGetLastError();
}

hipError_t launch_penalize_logits(const LogitsParams& p, hipStream_t s)
{
    // Short slices fill the chip where rows are few, long ones read a row's history fewer times.
    auto go = [&](auto rounds) {
        constexpr int R = decltype(rounds)::value;
        const long long slices = (p.vocab + slice_tokens(R) - 1) / slice_tokens(R);
        const dim3 grid((unsigned)((p.rows + 7) / 8 * 8 * slices));
        if (p.bf16)
            hipLaunchKernelGGL((penalize_kernel<true, R>), grid, dim3(kThreads), 0, s, p, (int)slices);
        else
            hipLaunchKernelGGL((penalize_kernel<false, R>), grid, dim3(kThreads), 0, s, p, (int)slices);
    };
    // Rows of 128256 tokens, slices of 2 / 4 / 8 rounds.  fp32, histories of 128 to 1024: 1 row 9.0 / 9.4 / 12.5 us, 16 rows
    // 9.7 / 10.8 / 13.8, 32 rows 15.0 / 15.1 / 17.2, 64 rows 20.8 / 19.6 / 21.0, 96 rows 27.5 / 25.5 / 24.4, 128 rows 34.3 / 30.8 / 32.9, of 4 / 8
    // rounds 256 rows 65.0 / 64.3, 1024 rows 211 / 203; bf16, histories up to 2048: 1024 rows 339 / 225 / 176.  Rows of 32000 fp32 tokens: 64 rows
    // 9.7 / 10.7 / 13.8, 1024 rows 75.6 / 64.6 / 67.6.  Rows shorter than a slice leave wavefronts without logits: 1024 rows of 4096 tokens
    // 15.1 / 16.5 / 22.7, 8192 rows of 1024 60 / 64 / 94 (the rule takes 4).
    const long long tokens = p.rows * p.vocab;
    if (tokens >= 12000000)
        go(std::integral_constant<int, 8>{});
    else if (tokens >= 3000000)
        go(std::integral_constant<int, 4>{});
    else
        go(std::integral_constant<int, 2>{});
    return hipGetLastError();
}

}  // namespace spd
