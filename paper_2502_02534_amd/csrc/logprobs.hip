// Log probabilities of given tokens, with rank, entropy and the most probable tokens: one workgroup a row.
//
// With d_i = (x_i - max x) / T (no overflow, whatever the logits), Z = sum exp(d_i):
//   log p_i = d_i - ln Z,  entropy = ln Z + sum exp(d_i) (-d_i) / Z  (both terms >= 0: nothing cancels)
#include "spd_internal.h"

#include <hip/hip_bfloat16.h>

namespace spd {
namespace {

constexpr int kThreads = 256;

template <bool BF16> __device__ __forceinline__ float logit(const LogprobsParams& p, long long at)
{
    if (BF16)
        return __uint_as_float((unsigned)((const unsigned short*)p.logits)[at] << 16);
    return ((const float*)p.logits)[at];
}

// Larger logits first, then the lower token: whole numbers in that order, all different.
__device__ __forceinline__ unsigned long long key_of(float x, unsigned i)
{
    const unsigned u = __float_as_uint(x == 0.f ? 0.f : x);
    return (unsigned long long)((u & 0x80000000u) ? ~u : (u | 0x80000000u)) << 32 | (0xffffffffu - i);
}

__device__ __forceinline__ float logit_of(unsigned long long key)
{
    const unsigned u = (unsigned)(key >> 32);
    return __uint_as_float((u & 0x80000000u) ? (u & 0x7fffffffu) : ~u);
}

template <class T, class F> __device__ T over_block(T v, T* lds, F join)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        v = join(v, (T)__shfl_xor(v, o));
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
    for (int w = 1; w < kThreads / 64; ++w)
        v = join(v, lds[w]);
    return v;
}

template <bool BF16> __global__ __launch_bounds__(kThreads) void logprobs_kernel(LogprobsParams p)
{
    __shared__ double lds_d[4];
    __shared__ unsigned long long lds_k[4];
    const long long row = blockIdx.x, base = row * p.stride;
    const int vocab = (int)p.vocab;
    const int token = p.tokens ? p.tokens[row] : -1;
    const bool known = token >= 0 && token < vocab;
    const float given = known ? logit<BF16>(p, base + token) : 0.f;
    const float t = p.temperature ? p.temperature[row] : 1.f;
    const float inv_t = t > 0.f ? 1.f / t : 1.f;
    float m = -INFINITY;
    int above = 0;
    for (int i = threadIdx.x; i < vocab; i += kThreads) {
        const float x = logit<BF16>(p, base + i);
        m = fmaxf(m, x);
        above += x > given;
    }
    m = (float)over_block<double>(m, lds_d, [](double a, double b) { return a > b ? a : b; });
    above = (int)over_block<double>(above, lds_d, [](double a, double b) { return a + b; });
    double z = 0., s = 0.;
    if (m > -INFINITY)
        for (int i = threadIdx.x; i < vocab; i += kThreads) {
            const float d = (logit<BF16>(p, base + i) - m) * inv_t, e = expf(d);
            z += e;
            s += e > 0.f ? e * -d : 0.f;
        }
    z = over_block<double>(z, lds_d, [](double a, double b) { return a + b; });
    s = over_block<double>(s, lds_d, [](double a, double b) { return a + b; });
    const bool empty = !(m > -INFINITY);
    const float log_z = empty ? 0.f : (float)log(z);
    const auto log_p = [&](float x) { return empty ? -INFINITY : (x - m) * inv_t - log_z; };
    if (threadIdx.x == 0) {
        if (p.logprobs)
            p.logprobs[row] = known ? log_p(given) : -INFINITY;
        if (p.ranks)
            p.ranks[row] = known ? above + 1 : 0;
        if (p.entropy)
            p.entropy[row] = empty ? 0.f : (float)(log(z) + s / z);
        if (p.lse)
            p.lse[row] = empty ? -INFINITY : m * inv_t + log_z;
    }
    unsigned long long last = ~0ull;
    for (int k = 0; k < p.top; ++k) {
        unsigned long long best = 0;
        for (int i = threadIdx.x; i < vocab; i += kThreads) {
            const unsigned long long key = key_of(logit<BF16>(p, base + i), i);
            if (key < last && key > best)
                best = key;
        }
        last = over_block<unsigned long long>(best, lds_k, [](unsigned long long a, unsigned long long b) { return a > b ? a : b; });
        if (threadIdx.x == 0) {
            if (p.top_tokens)
                p.top_tokens[row * p.top + k] = (int)(0xffffffffu - (unsigned)last);
            if (p.top_logprobs)
                p.top_logprobs[row * p.top + k] = log_p(logit_of(last));
        }
    }
}

}  // namespace

hipError_t launch_token_logprobs(const LogprobsParams& p, hipStream_t s)
{
    if (p.bf16)
        hipLaunchKernelGGL((logprobs_kernel<true>), dim3((unsigned)p.rows), dim3(kThreads), 0, s, p);
    else
        hipLaunchKernelGGL((logprobs_kernel<false>), dim3((unsigned)p.rows), dim3(kThreads), 0, s, p);
    return hipGetLastError();
}

}  // namespace spd
