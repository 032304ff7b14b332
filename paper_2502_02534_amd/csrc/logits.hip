// What stands between the logits and the sampler: which tokens a prompt holds (a bit per token of the vocabulary),
// and the logits shaped by penalties, biases and a grammar mask.
#include "spd_internal.h"

namespace spd {
namespace {

// ---- which tokens occur in a prompt ----------------------------------------------------------------------
// One workgroup per prompt and stretch of the vocabulary: the stretch's bits are collected in LDS.
constexpr int kMarkThreads = 1024;
constexpr int kMarkWords = 4096;  // of a stretch (131072 tokens)

__global__ __launch_bounds__(kMarkThreads) void mark_tokens_kernel(const int* tokens, const int* indptr, long long vocab,
                                                                   uint32_t* bits, long long stride, int accumulate)
{
    __shared__ uint32_t lds[kMarkWords];
    const long long all_words = (vocab + 31) / 32, word0 = (long long)blockIdx.y * kMarkWords;
    const int words = (int)min(all_words - word0, (long long)kMarkWords);
    uint32_t* row = bits + (long long)blockIdx.x * stride + word0;
    for (int w = threadIdx.x; w < words; w += kMarkThreads)
        lds[w] = accumulate ? row[w] : 0u;
    __syncthreads();
    const long long lo = word0 * 32, hi = min(vocab, lo + (long long)words * 32);
    for (int t = indptr[blockIdx.x] + (int)threadIdx.x, end = indptr[blockIdx.x + 1]; t < end; t += kMarkThreads) {
        const int id = tokens[t];
        if (id >= lo && id < hi)
            atomicOr(&lds[(id - lo) >> 5], 1u << (id & 31));
    }
    __syncthreads();
    for (int w = threadIdx.x; w < words; w += kMarkThreads)
        row[w] = lds[w];
}

// ---- penalties, biases, grammar mask -----------------------------------------------------------------------
// One workgroup per row and slice of the vocabulary.  The row's generated tokens that lie in the slice are
// counted in LDS, then the slice's logits pass through once; biases, few, are added in LDS beforehand.
constexpr int kThreads = 256;
constexpr int kSlice = 4096;

__global__ __launch_bounds__(kThreads) void penalize_kernel(LogitsParams p, int slices)
{
    __shared__ uint32_t counts[kSlice];
    __shared__ float bias[kSlice];
    const long long r = blockIdx.x / slices;
    const long long i0 = (long long)(blockIdx.x % slices) * kSlice;
    const int len = (int)min((long long)kSlice, p.vocab - i0);
    for (int i = threadIdx.x; i < kSlice; i += kThreads) {
        counts[i] = 0u;
        bias[i] = 0.f;
    }
    __syncthreads();
    if (p.tokens) {
        const int n = min(p.token_lens[r], p.max_tokens);
        const int* mine = p.tokens + r * p.token_row_stride;
        for (int t = threadIdx.x; t < n; t += kThreads) {
            const long long id = mine[t * p.token_step_stride] - i0;
            if (id >= 0 && id < len)
                atomicAdd(&counts[id], 1u);
        }
    }
    if (p.bias_tokens)
        for (int b = p.bias_indptr[r] + (int)threadIdx.x, end = p.bias_indptr[r + 1]; b < end; b += kThreads) {
            const long long id = p.bias_tokens[b] - i0;
            if (id >= 0 && id < len)
                bias[id] = p.bias_values[b];
        }
    __syncthreads();
    const float rep = p.repetition ? p.repetition[r] : 1.f;
    const float freq = p.frequency ? p.frequency[r] : 0.f, pres = p.presence ? p.presence[r] : 0.f;
    const long long prompt = !p.prompt_bits ? -1 : p.prompt_of_row ? p.prompt_of_row[r] : r;
    const long long grammar = !p.allowed_bits ? -1 : p.allowed_of_row ? p.allowed_of_row[r] : r;
    const uint32_t* seen_words = p.prompt_bits + (prompt < 0 ? 0 : prompt) * p.prompt_stride;
    const uint32_t* allowed_words = p.allowed_bits + (grammar < 0 ? 0 : grammar) * p.allowed_stride;
    for (int k = threadIdx.x; k < len; k += kThreads) {
        const long long i = i0 + k;
        float x = p.bf16 ? __uint_as_float((uint32_t)((const uint16_t*)p.logits)[r * p.stride + i] << 16)
                         : ((const float*)p.logits)[r * p.stride + i];
        const uint32_t c = counts[k];
        if (c != 0u || (prompt >= 0 && ((seen_words[i >> 5] >> (i & 31)) & 1u)))
            x = x > 0.f ? x / rep : x * rep;
        if (c != 0u)
            x = x - freq * (float)c - pres;
        x += bias[k];
        if (grammar >= 0 && !((allowed_words[i >> 5] >> (i & 31)) & 1u))
            x = -INFINITY;
        p.out[r * p.out_stride + i] = x;
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
    const long long slices = (p.vocab + kSlice - 1) / kSlice;
    hipLaunchKernelGGL(penalize_kernel, dim3((unsigned)(p.rows * slices)), dim3(kThreads), 0, s, p, (int)slices);
    return hipGetLastError();
}

}  // namespace spd
