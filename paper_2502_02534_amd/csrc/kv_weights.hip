// How much of the queries' attention every cached token got:
//   w'[b, j, t] = decay w[b, j, t] + sum over the query rows (i, h) that see t of 2^(scale_log2 q . k_t - lse_log2)
// One workgroup takes 64 tokens of one KV head and all query rows of their sequence, so a weight has one owner and its
// sum one order.
#include "spd_internal.h"

namespace spd {
namespace {

constexpr int kThreads = 256, kTokens = 64;

template <bool BF16> __device__ __forceinline__ float element(const void* x, long long at)
{
    if (BF16)
        return __uint_as_float((unsigned)((const unsigned short*)x)[at] << 16);
    return ((const float*)x)[at];
}

template <bool BF16> __global__ __launch_bounds__(kThreads) void kv_weights_kernel(KvWeightsParams p, int tiles)
{
    __shared__ float sums[4][kTokens];
    const int j = blockIdx.x % p.Hkv, tile = blockIdx.x / p.Hkv % tiles, b = blockIdx.x / p.Hkv / tiles;
    const int L = min(p.kv_lens[b], p.max_kv), t0 = tile * kTokens;
    if (t0 >= L)
        return;
    const int q0 = p.query_indptr[b], n = min(p.query_indptr[b + 1] - q0, p.max_query);
    const int part = threadIdx.x >> 6, t = t0 + (threadIdx.x & 63), tk = min(t, L - 1), kv0 = p.kv_indptr[b];
    const long long k_at = p.page_size ? (((long long)p.pages[kv0 + tk / 16] * p.Hkv + j) * 16 + tk % 16) * p.D
                                       : (long long)(kv0 + tk) * p.kv_stride + (long long)j * p.D;
    float sum = 0.f;
    for (int r = part; r < n * p.G; r += 4) {
        const int i = r / p.G, h = j * p.G + r % p.G;
        const float lse = p.lse[(long long)(q0 + i) * p.Hq + h];
        if (lse == -INFINITY || (p.causal && t > L - n + i))
            continue;
        const long long q_at = (long long)(q0 + i) * p.q_stride + (long long)h * p.D;
        float s = 0.f;
        for (int c = 0; c < p.D; ++c)
            s = __builtin_fmaf(element<BF16>(p.q, q_at + c), element<BF16>(p.k, k_at + c), s);
        sum += __builtin_amdgcn_exp2f(__builtin_fmaf(s, p.scale_log2, -lse * kLog2e));
    }
    sums[part][threadIdx.x & 63] = sum;
    __syncthreads();
    if (part == 0 && t < L) {
        const long long at = ((long long)b * p.Hkv + j) * p.stride + t;
        const float all = (sums[0][threadIdx.x] + sums[1][threadIdx.x]) + (sums[2][threadIdx.x] + sums[3][threadIdx.x]);
        p.weights_out[at] = p.weights ? __builtin_fmaf(p.decay, p.weights[at], all) : all;
    }
}

}  // namespace

hipError_t launch_kv_weights(const KvWeightsParams& p, hipStream_t s)
{
    const int tiles = (p.max_kv + kTokens - 1) / kTokens;
    const dim3 grid((unsigned)((long long)tiles * p.Hkv * p.B));
    if (p.dtype == 1)
        hipLaunchKernelGGL((kv_weights_kernel<true>), grid, dim3(kThreads), 0, s, p, tiles);
    else
        hipLaunchKernelGGL((kv_weights_kernel<false>), grid, dim3(kThreads), 0, s, p, tiles);
    return hipGetLastError();
}

}  // namespace spd
