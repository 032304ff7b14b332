// Stores the keys and values of a batch of new tokens in the cache, each token's row at its slot: the copy between
// a prompt's projection and its attention.  A thread moves 16-byte pieces; bound by HBM (read and write once).
#include "spd_internal.h"

namespace spd {
namespace {

constexpr int kThreads = 256;
constexpr int kPerThread = 4;  // pieces of K and of V

__global__ __launch_bounds__(kThreads) void kv_write_kernel(KvWriteParams p)
{
    const unsigned row_u4 = (unsigned)(p.Hkv * p.head_u4);
    const long long total = p.tokens * row_u4;
    uint4 k[kPerThread], v[kPerThread];
    long long to[kPerThread];
#pragma unroll
    for (int u = 0; u < kPerThread; ++u) {
        const long long i = ((long long)blockIdx.x * kPerThread + u) * kThreads + threadIdx.x;
        to[u] = -1;
        if (i < total) {
            const long long t = i / row_u4;
            const unsigned c = (unsigned)(i - t * row_u4);
            k[u] = ((const uint4*)p.k)[t * p.stride_u4 + c];
            v[u] = ((const uint4*)p.v)[t * p.stride_u4 + c];
            const long long slot = p.slots[t];
            if (slot >= 0 && slot < p.num_slots) {
                if (p.page_size == 0)
                    to[u] = slot * row_u4 + c;
                else
                    to[u] = ((slot / p.page_size * p.Hkv + c / p.head_u4) * p.page_size + slot % p.page_size) * p.head_u4 + c % p.head_u4;
            }
        }
    }
#pragma unroll
    for (int u = 0; u < kPerThread; ++u)
        if (to[u] >= 0) {
            ((uint4*)p.k_pool)[to[u]] = k[u];
            ((uint4*)p.v_pool)[to[u]] = v[u];
        }
}

}  // namespace

hipError_t launch_kv_write(const KvWriteParams& p, hipStream_t s)
{
    const long long per_block = (long long)kThreads * kPerThread, total = p.tokens * p.Hkv * p.head_u4;
    hipLaunchKernelGGL(kv_write_kernel, dim3((unsigned)((total + per_block - 1) / per_block)), dim3(kThreads), 0, s, p);
    return hipGetLastError();
}

}  // namespace spd
