// Attention of a batch of prompts' new tokens over their KV, causal or not: the kernel for fp32 (prompt_mfma.hip holds
// the one for bf16) and the joining of parts.
//
// The rows of a prompt and KV head are its (new token, query head of the group) pairs, token by token, so
// that the heads that share K and V share a tile.  Workgroup = (unit, KV head), a unit being 128 rows and a part of the
// tokens they see (prompt_units.h); a wavefront owns 32 rows and walks the tokens in tiles of 32 with the online softmax
// of the paper's attention tasks (App., attn task 2: running maximum, running sum, deferred division).
//
// Both products run on the matrix pipe in the transposed form S^T = K Q^T, O^T += V^T P^T, so that a lane
// owns one row in both: the softmax statistics are the lane's own (two lanes share a row's tokens) and P is the
// S^T accumulator itself (v_mfma_f32_32x32x2_f32: nothing is rounded to fewer bits).
//
// What a row must not see enters nowhere: scores are replaced, not added to, and where a tile holds tokens that
// some of its rows do not see and values that are not finite (0 * inf is not 0), these are taken out of the tile and
// added at the end to the rows that see them.
//
// Bound: the matrix pipe, 155 TFLOP/s for fp32 products.  The tile after the present one is on its way into registers
// while its products run, and goes to the other half of LDS after them: one barrier a tile (two: 4096 tokens 697 us, one: 582).
// 16 query and 4 KV heads, causal: 4096 tokens of 128 channels 582 us, 118 TFLOP/s of the products that the rows need (8192: 2.36 ms, 117),
// 8192 of 64 1.24 ms, 111; 8 and 4 heads, 2000 of 256 245 us, 67 (one workgroup a CU: its 134 KB of LDS leave no room for a second).
// Few rows: 256 tokens of 4 and 1 heads of 64 channels 9.0 us in 64 units of 32 tokens, and 3.4 for the launch that joins them.
#include "prompt_units.h"

#include <type_traits>

namespace spd {
namespace {

using prompt_impl::find_unit;
using prompt_impl::kRows;
using prompt_impl::Unit;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

constexpr int kTileN = 32;      // tokens per tile
constexpr int kThreads = 256;
// Tiles that some row of a workgroup does not see whole: its 128 rows end at up to 128 tokens, and a prompt's end may be ragged.
constexpr int kOddWords = 8;
constexpr float kNever = -3.402823466e38f;  // reference maximum of a row that has seen nothing: finite, so that no exponent is inf - inf

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const f32x2 v = {lo, hi};
    const bf16x2 r = __builtin_convertvector(v, bf16x2);
    return *reinterpret_cast<const uint32_t*>(&r);
}

// Zeroes the values of a piece that are not finite; whether there were any.
__device__ __forceinline__ bool take_odd(uint4& v)
{
    uint32_t* w = reinterpret_cast<uint32_t*>(&v);
    bool any = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool odd = (w[i] & 0x7f800000u) == 0x7f800000u;
        w[i] = odd ? 0u : w[i];
        any = any || odd;
    }
    return any;
}

template <int DP, bool PAGED>  // channels, padded with zeros
__global__ __launch_bounds__(kThreads, DP <= 128 ? 2 : 1) void prompt_attn_f32_kernel(PromptParams p)
{
    constexpr int kRowPieces = DP / 4, kPieces = kTileN * kRowPieces / kThreads;
    static_assert(kPieces * kThreads == kTileN * kRowPieces, "whole pieces per thread");
    // bytes between token rows: 16 lanes' equal pieces of K, and rows four apart of V, lie in different banks
    constexpr int kStrideK = DP * 4 + 16, kStrideV = DP * 4 + 32;
    __shared__ __align__(16) char lds_k[2][kTileN * kStrideK];
    __shared__ __align__(16) char lds_v[2][kTileN * kStrideV];
    __shared__ uint32_t lds_odd[kOddWords];  // tokens whose values are not all finite, a word per tile that some row does not see whole

    const int j = blockIdx.x % p.Hkv;
    const Unit at = find_unit(p, blockIdx.x / p.Hkv);
    if (!at.any)
        return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, h = lane >> 5;
    const int q0 = at.q0, n = at.n, L = at.L;
    const int row0 = at.tile * kRows, rr = row0 + wave * 32 + col;
    const bool row_ok = rr < n * p.G;
    const int token = (row_ok ? rr : 0) / p.G, head = j * p.G + (row_ok ? rr : 0) % p.G;
    // the last token a row sees, and the first and last row's
    const int limit = !row_ok ? -1 : p.causal ? L - n + token : L - 1;
    const int last_row = min(row0 + kRows, n * p.G) - 1;
    const int least = p.causal ? L - n + row0 / p.G : L - 1, most = p.causal ? L - n + last_row / p.G : L - 1;
    const int wave_last = min(row0 + wave * 32 + 32, n * p.G) - 1;
    const int wave_most = wave_last < row0 + wave * 32 ? -1 : p.causal ? L - n + wave_last / p.G : L - 1;

    // this part's tokens
    const int seen = max(most + 1, 0);
    const int t0 = p.num_splits > 1 ? min(at.split * at.split_tokens, seen) : 0;
    const int t1 = p.num_splits > 1 ? min(t0 + at.split_tokens, seen) : seen;

    const int first = at.kv0;
    auto offset = [&](int t) -> long long {  // of token t's row of this KV head, in bytes
        if (PAGED)
            return (((long long)p.pages[first + (t >> 4)] * p.Hkv + j) * 16 + (t & 15)) * p.D * 4;
        return ((long long)(first + t) * p.kv_stride + (long long)j * p.D) * 4;
    };
    uint4 kreg[kPieces], vreg[kPieces];
    int page[kPieces] = {};  // of the tile that is requested next: asked for a tile ahead where the registers allow
    auto fetch_pages = [&](int tb) __attribute__((always_inline)) {
        if (PAGED) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
                page[i] = p.pages[first + (min(tb + (tid + i * kThreads) / kRowPieces, t1 - 1) >> 4)];
        }
    };
    auto request = [&](int tb) __attribute__((always_inline)) {
        if (DP > 128)
            fetch_pages(tb);
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int piece = tid + i * kThreads, row = piece / kRowPieces, c = piece % kRowPieces, t = tb + row;
            kreg[i] = vreg[i] = make_uint4(0u, 0u, 0u, 0u);
            if (t < t1 && c * 4 < p.D) {
                const long long o = c * 16 + (PAGED ? (((long long)page[i] * p.Hkv + j) * 16 + (t & 15)) * p.D * 4
                                                : ((long long)(first + t) * p.kv_stride + (long long)j * p.D) * 4);
                kreg[i] = *reinterpret_cast<const uint4*>((const char*)p.k + o);
                vreg[i] = *reinterpret_cast<const uint4*>((const char*)p.v + o);
            }
        }
        if (DP <= 128)
            fetch_pages(tb + kTileN);
    };
    const int whole = max(min(least + 1, t1) - t0, 0) / kTileN;  // tiles that every row sees whole
    auto put = [&](int nth) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int piece = tid + i * kThreads, row = piece / kRowPieces, c = piece % kRowPieces;
            if (nth >= whole && take_odd(vreg[i]))
                atomicOr(&lds_odd[min(nth - whole, kOddWords - 1)], 1u << row);
            *reinterpret_cast<uint4*>(lds_k[nth & 1] + row * kStrideK + c * 16) = kreg[i];
            *reinterpret_cast<uint4*>(lds_v[nth & 1] + row * kStrideV + c * 16) = vreg[i];
        }
    };
    if (t0 < t1) {
        fetch_pages(t0);
        request(t0);
    }
    // Channels 8 u + 4 h .. + 3 of the lane's row, with the scale (one more rounding of 2^-24 a term): scores come out in base 2, and the
    // highest of a row is the reference maximum to the last bit however large it is (a scale within the exponent's fma would leave
    // the product's rounding, more than an exponent holds from 2^31 on).
    floatx4 qf[DP / 8];
    {
        const float* q = (const float*)p.q + (long long)(q0 + token) * p.q_stride + (long long)head * p.D;
#pragma unroll
        for (int u = 0; u < DP / 8; ++u) {
            floatx4 v = {0.f, 0.f, 0.f, 0.f};
            if (8 * u + 4 * h < p.D)
                v = *reinterpret_cast<const floatx4*>(q + 8 * u + 4 * h);
            qf[u] = v * p.scale_log2;
        }
    }

    float m = kNever, l = 0.f;
    floatx16 o[DP / 32];
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i)
            o[db][i] = 0.f;

    if (tid < kOddWords)
        lds_odd[tid] = 0u;
    __syncthreads();
    if (t0 < t1)
        put(0);
#pragma unroll
    for (int u = 0; DP <= 128 && u < DP / 8; ++u)  // waits for the queries here: a wait in the loop would be for the next tile's loads too
        asm volatile("" : "+v"(qf[u]));
    __syncthreads();
    int nth = 0;
    for (int tb = t0; tb < t1; tb += kTileN, ++nth) {
        if (tb + kTileN < t1)
            request(tb + kTileN);
        if (tb <= wave_most) {
            const char* const k = lds_k[nth & 1] + col * kStrideK + 16 * h;
            const char* const v = lds_v[nth & 1] + 4 * h * kStrideV + col * 4;
            floatx16 s = {};
            floatx4 a = *reinterpret_cast<const floatx4*>(k);
#pragma unroll
            for (int u = 0; u < DP / 8; ++u) {
                const floatx4 now = a;
                if (u + 1 < DP / 8)
                    a = *reinterpret_cast<const floatx4*>(k + (u + 1) * 32);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    s = __builtin_amdgcn_mfma_f32_32x32x2f32(now[i], qf[u][i], s, 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);  // (all the reads ahead of all the products would not fit the registers)
            }
            // accumulator register i of lane-half h is token 8 (i/4) + 4 h + i%4 of the tile
            if (nth >= whole) {  // some row does not see all of the tile
                const int end = min(limit, t1 - 1) - tb - 4 * h;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    s[i] = 8 * (i >> 2) + (i & 3) <= end ? s[i] : -INFINITY;
            }
            float top = s[0];
#pragma unroll
            for (int i = 1; i < 16; ++i)
                top = fmaxf(top, s[i]);
            top = fmaxf(top, __shfl_xor(top, 32));
            // the reference maximum only has to bound the exponents: raised where the tile's is well above it
            if (__ballot(top > m + 10.f) != 0) {
                const float m_new = fmaxf(m, top), corr = __builtin_amdgcn_exp2f(m - m_new);
                m = m_new;
                l *= corr;
#pragma unroll
                for (int db = 0; db < DP / 32; ++db) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        o[db][i] *= corr;
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[i] = __builtin_amdgcn_exp2f(s[i] - m);
                sum += s[i];
            }
            l += sum;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const char* row = v + (8 * (i >> 2) + (i & 3)) * kStrideV;
#pragma unroll
                for (int db = 0; db < DP / 32; ++db)
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(*reinterpret_cast<const float*>(row + 128 * db), s[i], o[db], 0, 0, 0);
                if (DP > 128 && (i & 1))
                    __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (tb + kTileN < t1)
            put(nth + 1);
        __syncthreads();
    }

    l += __shfl_xor(l, 32);
    if (!row_ok)
        return;
    const long long row = (long long)(q0 + token) * p.Hq + head;
    float inv = 1.f;
    float* dst = (float*)p.out + row * p.D;
    if (p.num_splits > 1) {
        if (h == 0) {
            p.part_ml[row * p.num_splits + at.split] = make_float4(m, l, 0.f, 0.f);
            if (at.split == 0)  // and the parts that this prompt does not have
                for (int s = at.splits; s < p.num_splits; ++s)
                    p.part_ml[row * p.num_splits + s] = make_float4(kNever, 0.f, 0.f, 0.f);
        }
        if (t0 >= t1)
            return;
        dst = (float*)p.part_acc + (row * p.num_splits + at.split) * p.D;
    } else {
        inv = l == 0.f ? 0.f : 1.f / l;
        if (p.lse && h == 0)
            p.lse[row] = l == 0.f ? -INFINITY : m * kLn2 + logf(l);
    }
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
            const int c = 32 * db + 8 * q4 + 4 * h;
            if (c < p.D)
                *reinterpret_cast<float4*>(dst + c) =
                    make_float4(o[db][4 * q4] * inv, o[db][4 * q4 + 1] * inv, o[db][4 * q4 + 2] * inv, o[db][4 * q4 + 3] * inv);
        }
    // rare: the values that were taken out of the tiles, to the rows that see them (a lane's own channels, as stored above)
    for (int w = 0; w < kOddWords; ++w)
        for (uint32_t bits = lds_odd[w]; bits != 0u; bits &= bits - 1u) {
            const int x = t0 + (whole + w) * kTileN + __ffs(bits) - 1;
            if (x >= t1 || x > limit)
                continue;
            const float* v = (const float*)((const char*)p.v + offset(x));
            for (int c0 = 4 * h; c0 < p.D; c0 += 8)
                for (int c = c0; c < c0 + 4; ++c)
                    if (!(fabsf(v[c]) < INFINITY))
                        dst[c] += v[c];
        }
}

// Joins the parts of a row: with states (m_i, l_i, acc_i), m = max m_i and w_i = 2^(m_i - m),
// out = sum w_i acc_i / sum w_i l_i.  LANES lanes take a part of a row, 16 bytes each, and SUB such groups
// every SUB-th part; each group also takes all its parts' (m, l) and hands their weights round.  Bound by latency, then by the
// partial states, whose loads a lane has in flight kBatch at a time:
// 7200 rows in 3 to 9 parts of 128 channels 8.2 us, 1024 rows of 128 channels in 32 parts 9.3 (17 MB), of 64 in 8 parts 3.5.
template <typename T, int LANES, int SUB>
__global__ __launch_bounds__(kThreads, 7) void prompt_merge_kernel(PromptParams p)
{
    constexpr int kRowsPerBlock = kThreads / (LANES * SUB), kBatch = SUB > 1 ? 4 : 8, kCh = 4;
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES % SUB, first_lane = (threadIdx.x & 63) - lane, c = lane * kCh;
    const long long row = (long long)blockIdx.x * kRowsPerBlock + threadIdx.x / (LANES * SUB);
    // (rows before the first prompt's and past the last one's have no states: they belong to nobody in this call)
    const bool row_ok = row >= (long long)p.query_indptr[0] * p.Hq && row < (long long)p.query_indptr[p.B] * p.Hq && row < p.rows;
    const int S = p.num_splits;
    const float4* ml = p.part_ml + (row_ok ? row : 0) * S;
    const char* parts = (const char*)p.part_acc + ((row_ok ? row : 0) * S * p.D + (c < p.D ? c : 0)) * 4;
    const long long part_bytes = (long long)p.D * 4;
    uint4 a[kBatch];
    auto request = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            a[k] = make_uint4(0u, 0u, 0u, 0u);
            if (s0 + group + SUB * k < S)
                a[k] = *reinterpret_cast<const uint4*>(parts + (s0 + group + SUB * k) * part_bytes);
        }
    };
    request(0);  // the first parts need not wait for their weights
    float m = -INFINITY;
    for (int s = lane; s < S; s += LANES) {
        const float4 x = ml[s];
        m = x.y != 0.f ? fmaxf(m, x.x) : m;
    }
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1)
        m = fmaxf(m, __shfl_xor(m, o));
    float l = 0.f, acc[kCh];
#pragma unroll
    for (int e = 0; e < kCh; ++e)
        acc[e] = 0.f;
    for (int s0 = 0; s0 < S; s0 += LANES) {  // LANES weights at a time
        float w = 0.f;
        if (s0 + lane < S) {
            const float4 x = ml[s0 + lane];
            if (x.y != 0.f) {  // (a sum that is not a number stays one)
                const float u = __builtin_amdgcn_exp2f(x.x - m);
                l = fmaf(u, x.y, l);
                w = u;
            }
        }
        // up to the last part that holds anything: a prompt may have fewer than the longest one
        const unsigned long long holds = __ballot(w != 0.f) >> first_lane;
        const int here = 64 - __clzll((long long)(LANES == 64 ? holds : holds & ((1ull << (LANES & 63)) - 1)));
#pragma unroll 1  // (rounds side by side would not fit the registers)
        for (int k0 = 0; k0 < here; k0 += SUB * kBatch) {
            if (s0 + k0 > 0)
                request(s0 + k0);
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int at = k0 + group + SUB * k;
                const float ws = __shfl(w, first_lane + min(at, LANES - 1));
                if (ws != 0.f && at < here) {  // (a part that holds nothing was not written)
                    const uint32_t v[4] = {a[k].x, a[k].y, a[k].z, a[k].w};
#pragma unroll
                    for (int e = 0; e < kCh; ++e)
                        acc[e] = fmaf(ws, __uint_as_float(v[e]), acc[e]);
                }
            }
        }
    }
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1)
        l += __shfl_xor(l, o);
#pragma unroll
    for (int o = LANES; o < LANES * SUB; o <<= 1)
#pragma unroll
        for (int e = 0; e < kCh; ++e)
            acc[e] += __shfl_xor(acc[e], o);
    if (!row_ok || group != 0)
        return;
    const bool none = l == 0.f;
    const float inv = none ? 0.f : 1.f / l;
    if (p.lse && lane == 0)
        p.lse[row] = none ? -INFINITY : m * kLn2 + logf(l);
    if (c >= p.D)
        return;
    char* dst = (char*)p.out + (row * p.D + c) * (long long)sizeof(T);
    if constexpr (sizeof(T) == 2)
        *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv));
    else
        *reinterpret_cast<float4*>(dst) = make_float4(acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
}

template <typename T, int LANES> void launch_merge(const PromptParams& p, hipStream_t s)
{
    // Few rows: a wavefront for each, so that all its parts are on their way at once.  One / several groups of lanes, whole calls: 32 new tokens of
    // 32 bf16 heads of 128 channels (1024 rows) over 2048 tokens 20.5 / 17.3 us, over 16384 36.4 / 32.3; two such prompts over 4096 (2048 rows)
    // 27.3 / 26.9, four (4096 rows) 34.4 / 34.2; 7200 rows in 3 to 9 (of up to 12) parts 46.3 / 47.1; 1024 fp32 rows of 64 in 8 parts 3.9 / 3.6 (the join alone).
    constexpr int kSub = 64 / LANES;
    const auto go = [&](auto sub) {
        constexpr int SUB = decltype(sub)::value, kRowsPerBlock = kThreads / (LANES * SUB);
        hipLaunchKernelGGL((prompt_merge_kernel<T, LANES, SUB>), dim3((unsigned)((p.rows + kRowsPerBlock - 1) / kRowsPerBlock)),
                           dim3(kThreads), 0, s, p);
    };
    if (kSub > 1 && p.rows <= 2048)
        go(std::integral_constant<int, kSub>{});
    else
        go(std::integral_constant<int, 1>{});
}

template <int DP, int LANES> void launch_f32(const PromptParams& p, hipStream_t s)
{
    const dim3 grid((unsigned)((long long)p.tiles * p.num_splits * p.Hkv)), block(kThreads);
    // Two workgroups a CU, which the pairs of tiles and the length of parts count on (prompt_units.h): 64 channels alone would fit
    // four, and then long units share a CU.  16 heads, 64 channels, with four / three / two a CU: 2 x 4096 tokens 654 / 606 / 634 us,
    // 1 x 8192 1284 / 1182 / 1241 (three are ahead where there are neither pairs nor parts).
    constexpr int kSpareLds = DP == 64 ? 20480 : 0;
    if (p.page_size != 0)
        hipLaunchKernelGGL((prompt_attn_f32_kernel<DP, true>), grid, block, kSpareLds, s, p);
    else
        hipLaunchKernelGGL((prompt_attn_f32_kernel<DP, false>), grid, block, kSpareLds, s, p);
    if (p.num_splits > 1)
        launch_merge<float, LANES>(p, s);
}

}  // namespace

hipError_t launch_prompt_attn(const PromptParams& p, hipStream_t s)
{
    if (p.dtype == 1) {
        const hipError_t e = launch_prompt_mfma(p, s);
        if (e != hipSuccess)
            return e;
        if (p.num_splits > 1)
            p.D <= 64 ? launch_merge<__bf16, 16>(p, s) : p.D <= 128 ? launch_merge<__bf16, 32>(p, s) : launch_merge<__bf16, 64>(p, s);
    } else {
        p.D <= 64 ? launch_f32<64, 16>(p, s) : p.D <= 128 ? launch_f32<128, 32>(p, s) : launch_f32<256, 64>(p, s);
    }
    return hipGetLastError();
}

}  // namespace spd
