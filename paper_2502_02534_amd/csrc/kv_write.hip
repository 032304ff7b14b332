// Stores the keys and values of a batch of new tokens in the cache, each token's row at its slot: the copy between
// a prompt's projection and its attention.
//
// Bound: HBM, each byte read and written once.  A thread moves one 16-byte piece of K and of V: 77.5k tokens of 8 bf16 heads of
// 128 channels in 110 us (5.2 TB/s; two pieces a thread 118, four 135, eight 175: the chip holds fewer rows open).
#include "spd_internal.h"

namespace spd {
namespace {

constexpr int kThreads = 256;

__global__ __launch_bounds__(kThreads) void kv_write_kernel(KvWriteParams p, unsigned head_magic)
{
    const unsigned row_u4 = (unsigned)(p.Hkv * p.head_u4);
    const unsigned long long i = (unsigned long long)blockIdx.x * kThreads + threadIdx.x;
    // (the division is exact in 32 bits where the pieces are that few)
    const unsigned long long t = i >> 32 ? i / row_u4 : (unsigned)i / row_u4;
    if (t >= (unsigned long long)p.tokens)
        return;
    const unsigned c = (unsigned)(i - t * row_u4);
    const long long from = (long long)t * p.stride_u4 + c, slot = p.slots[t];
    const uint4 k = ((const uint4*)p.k)[from], v = ((const uint4*)p.v)[from];
    if (slot < 0 || slot >= p.num_slots)
        return;
    const unsigned head = head_magic != 0u ? __umulhi(c, head_magic) : c, in_head = c - head * (unsigned)p.head_u4;
    const long long to = p.page_size == 0 ? slot * row_u4 + c : (((slot >> 4) * p.Hkv + head) * 16 + (slot & 15)) * p.head_u4 + in_head;
    ((uint4*)p.k_pool)[to] = k;
    ((uint4*)p.v_pool)[to] = v;
}

}  // namespace

hipError_t launch_kv_write(const KvWriteParams& p, hipStream_t s)
{
    const long long total = p.tokens * p.Hkv * p.head_u4;
    // c / head_u4 = umulhi(c, 2^32 / head_u4 + 1) for c < 2^32 / head_u4 (a row has at most 2^22 pieces, a head 64)
    const unsigned magic = p.head_u4 > 1 ? (unsigned)((1ull << 32) / p.head_u4 + 1) : 0u;
    hipLaunchKernelGGL(kv_write_kernel, dim3((unsigned)((total + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, p, magic);
    return hipGetLastError();
}

}  // namespace spd
