// Attention of a batch of prompts' new tokens over their KV, causal or not.
//
// The rows of a prompt and KV head are its (new token, query head of the group) pairs, token by token, so
// that the heads that share K and V share a tile.  Workgroup = (tile of 128 rows, KV head, split of the tokens
// the tile sees); a wavefront owns 32 rows and walks the tokens in tiles of 32 with the online softmax of the
// paper's attention tasks (App., attn task 2: running maximum, running sum, deferred division).
//
// Both products run on the matrix pipe in the transposed form S^T = K Q^T, O^T += V^T P^T, so that a lane
// owns one row in both: the softmax statistics are the lane's own (two lanes share a row's tokens) and P is the
// S^T accumulator itself.  bf16: v_mfma_f32_32x32x16_bf16, P rounded to bf16 (its 2^-9 is that of the
// result's own rounding; the sum l takes the unrounded values).  fp32: v_mfma_f32_32x32x2_f32, nothing rounded.
//
// What a row must not see enters nowhere: scores are replaced, not added to, and where a tile holds tokens that
// some of its rows do not see and values that are not finite (0 * inf is not 0), its tokens are added one by
// one, each to the rows that see it.
#include "prompt_units.h"

#include <hip/hip_fp16.h>

namespace spd {
namespace {

using prompt_impl::find_unit;
using prompt_impl::kRows;
using prompt_impl::Unit;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

constexpr int kTileN = 32;      // tokens per tile
constexpr int kThreads = 256;

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const f32x2 v = {lo, hi};
    const bf16x2 r = __builtin_convertvector(v, bf16x2);
    return *reinterpret_cast<const uint32_t*>(&r);
}

// Operands of the two products for an element type; a piece is 16 bytes.
template <typename T, int DP> struct Mat;

template <int DP> struct Mat<__bf16, DP> {
    static constexpr int kStrideK = DP * 2 + 16, kStrideV = DP * 2 + 16;  // bytes between token rows in LDS
    bf16x8 qf[DP / 16];  // channels 16 s + 8 h .. + 7 of the lane's row
    __device__ __forceinline__ void load_q(const char* row, int d, int h, bool ok)
    {
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) {
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (ok && 16 * s + 8 * h < d)
                v = *reinterpret_cast<const uint4*>(row + (16 * s + 8 * h) * 2);
            qf[s] = *reinterpret_cast<bf16x8*>(&v);
        }
    }
    __device__ __forceinline__ floatx16 scores(const char* k, int col, int h) const
    {
        floatx16 s = {};
#pragma unroll
        for (int u = 0; u < DP / 16; ++u) {
            const bf16x8 a = *reinterpret_cast<const bf16x8*>(k + col * kStrideK + (16 * u + 8 * h) * 2);
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[u], s, 0, 0, 0);
        }
        return s;
    }
    __device__ __forceinline__ void add_values(const char* v, const floatx16& pr, floatx16 (&o)[DP / 32], int lane) const
    {
        const int h = lane >> 5, g16 = (lane >> 4) & 1, r = (lane & 15) >> 2, q4 = lane & 3;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            const uint4 w = make_uint4(pack_bf16(pr[8 * ks], pr[8 * ks + 1]), pack_bf16(pr[8 * ks + 2], pr[8 * ks + 3]),
                                       pack_bf16(pr[8 * ks + 4], pr[8 * ks + 5]), pack_bf16(pr[8 * ks + 6], pr[8 * ks + 7]));
            const bf16x8 b = *reinterpret_cast<const bf16x8*>(&w);
#pragma unroll
            for (int db = 0; db < DP / 32; ++db) {
                // the transposing read hands each lane four tokens of one channel
                union {
                    shortx4 part[2];
                    bf16x8 all;
                } a;
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    const char* at = v + (16 * ks + 8 * part + 4 * h + r) * kStrideV + (32 * db + 16 * g16 + 4 * q4) * 2;
                    a.part[part] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (__attribute__((address_space(3))) shortx4*)(size_t)(__attribute__((address_space(3))) const void*)at);
                }
                o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.all, b, o[db], 0, 0, 0);
            }
        }
    }
    // Whether a piece holds values that are not finite.
    static __device__ __forceinline__ bool odd(const uint4& v)
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        bool any = false;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            any = any || (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
        return any;
    }
    // Token x of the tile alone, to the rows (lanes) that see it.
    __device__ __forceinline__ void add_token(const char* v, const floatx16& pr, floatx16 (&o)[DP / 32], int lane, int x, bool seen) const
    {
        const int h = lane >> 5, col = lane & 31, slot = (x >> 3) * 4 + (x & 3);  // accumulator register of the token
        float mine = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            mine = i == slot ? pr[i] : mine;
        const bool own = h == ((x >> 2) & 1);
        const uint4 w = make_uint4(own ? pack_bf16(mine, 0.f) : 0u, 0u, 0u, 0u);
#pragma unroll
        for (int db = 0; db < DP / 32; ++db) {
            const uint4 a = make_uint4(own ? *reinterpret_cast<const uint16_t*>(v + x * kStrideV + (32 * db + col) * 2) : 0u, 0u, 0u, 0u);
            const floatx16 t = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(&a),
                                                                       *reinterpret_cast<const bf16x8*>(&w), o[db], 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 16; ++i)
                o[db][i] = seen ? t[i] : o[db][i];
        }
    }
};

template <int DP> struct Mat<float, DP> {
    static constexpr int kStrideK = DP * 4 + 16, kStrideV = DP * 4 + 32;
    floatx4 qf[DP / 8];  // channels 8 u + 4 h .. + 3
    __device__ __forceinline__ void load_q(const char* row, int d, int h, bool ok)
    {
#pragma unroll
        for (int u = 0; u < DP / 8; ++u) {
            floatx4 v = {0.f, 0.f, 0.f, 0.f};
            if (ok && 8 * u + 4 * h < d)
                v = *reinterpret_cast<const floatx4*>(row + (8 * u + 4 * h) * 4);
            qf[u] = v;
        }
    }
    __device__ __forceinline__ floatx16 scores(const char* k, int col, int h) const
    {
        floatx16 s = {};
#pragma unroll
        for (int u = 0; u < DP / 8; ++u) {
            const floatx4 a = *reinterpret_cast<const floatx4*>(k + col * kStrideK + (8 * u + 4 * h) * 4);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                s = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], qf[u][i], s, 0, 0, 0);
        }
        return s;
    }
    __device__ __forceinline__ void add_values(const char* v, const floatx16& pr, floatx16 (&o)[DP / 32], int lane) const
    {
        const int h = lane >> 5, col = lane & 31;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const char* row = v + (8 * (i >> 2) + 4 * h + (i & 3)) * kStrideV + col * 4;
#pragma unroll
            for (int db = 0; db < DP / 32; ++db)
                o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(*reinterpret_cast<const float*>(row + 128 * db), pr[i], o[db], 0, 0, 0);
        }
    }
    static __device__ __forceinline__ bool odd(const uint4& v)
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        bool any = false;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            any = any || (w[i] & 0x7f800000u) == 0x7f800000u;
        return any;
    }
    __device__ __forceinline__ void add_token(const char* v, const floatx16& pr, floatx16 (&o)[DP / 32], int lane, int x, bool seen) const
    {
        const int h = lane >> 5, col = lane & 31, slot = (x >> 3) * 4 + (x & 3);
        float mine = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            mine = i == slot ? pr[i] : mine;
        const bool own = h == ((x >> 2) & 1);
        mine = own ? mine : 0.f;
#pragma unroll
        for (int db = 0; db < DP / 32; ++db) {
            const float a = own ? *reinterpret_cast<const float*>(v + x * kStrideV + (32 * db + col) * 4) : 0.f;
            const floatx16 t = __builtin_amdgcn_mfma_f32_32x32x2f32(a, mine, o[db], 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 16; ++i)
                o[db][i] = seen ? t[i] : o[db][i];
        }
    }
};

template <typename T, int DP>
__global__ __launch_bounds__(kThreads) void prompt_attn_kernel(PromptParams p)
{
    using M = Mat<T, DP>;
    constexpr int E = sizeof(T), kRowPieces = DP * E / 16, kPieces = kTileN * kRowPieces / kThreads;
    static_assert(kPieces * kThreads == kTileN * kRowPieces, "whole pieces per thread");
    __shared__ __align__(16) char lds_k[kTileN * M::kStrideK];
    __shared__ __align__(16) char lds_v[kTileN * M::kStrideV];
    __shared__ uint32_t lds_odd[2];  // whether a tile holds values that are not finite

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

    // this part's tokens
    const int seen = max(most + 1, 0);
    const int t0 = p.num_splits > 1 ? min(at.split * at.split_tokens, seen) : 0;
    const int t1 = p.num_splits > 1 ? min(t0 + at.split_tokens, seen) : seen;

    M mat;
    mat.load_q((const char*)p.q + ((long long)(q0 + token) * p.q_stride + (long long)head * p.D) * E, p.D, h, row_ok);

    const int first = at.kv0;
    auto offset = [&](int t) -> long long {  // of token t's row of this KV head, in bytes
        if (p.page_size != 0)
            return (((long long)p.pages[first + (t >> 4)] * p.Hkv + j) * 16 + (t & 15)) * p.D * E;
        return ((long long)(first + t) * p.kv_stride + (long long)j * p.D) * E;
    };
    uint4 kreg[kPieces], vreg[kPieces];
    auto request = [&](int tb) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int piece = tid + i * kThreads, row = piece / kRowPieces, c = piece % kRowPieces;
            kreg[i] = vreg[i] = make_uint4(0u, 0u, 0u, 0u);
            if (tb + row < t1 && c * 16 < p.D * E) {
                const long long o = offset(tb + row) + c * 16;
                kreg[i] = *reinterpret_cast<const uint4*>((const char*)p.k + o);
                vreg[i] = *reinterpret_cast<const uint4*>((const char*)p.v + o);
            }
        }
    };

    float m = -INFINITY, l = 0.f;
    floatx16 o[DP / 32];
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i)
            o[db][i] = 0.f;

    if (tid < 2)
        lds_odd[tid] = 0u;
    if (t0 < t1)
        request(t0);
    int stage = 0;
    for (int tb = t0; tb < t1; tb += kTileN, stage ^= 1) {
        const bool masked = tb + kTileN - 1 > least;  // some row does not see all of the tile
        __syncthreads();  // everybody is done with the tile before
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int piece = tid + i * kThreads, row = piece / kRowPieces, c = piece % kRowPieces;
            if (masked && M::odd(vreg[i]))
                lds_odd[stage] = 1u;
            *reinterpret_cast<uint4*>(lds_k + row * M::kStrideK + c * 16) = kreg[i];
            *reinterpret_cast<uint4*>(lds_v + row * M::kStrideV + c * 16) = vreg[i];
        }
        __syncthreads();
        if (tb + kTileN < t1)
            request(tb + kTileN);
        if (tid == 0)
            lds_odd[stage ^ 1] = 0u;
        floatx16 s = mat.scores(lds_k, col, h);
        // accumulator register i of lane-half h is token 8 (i/4) + 4 h + i%4 of the tile
        if (masked || tb + kTileN > t1) {
            const int end = min(limit, t1 - 1) - tb - 4 * h;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                s[i] = 8 * (i >> 2) + (i & 3) <= end ? s[i] : -INFINITY;
        }
        float most_s = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i)
            most_s = fmaxf(most_s, s[i]);
        most_s = fmaxf(most_s, __shfl_xor(most_s, 32));
        const float m_new = fmaxf(m, most_s * p.scale_log2);
        const float ref = m_new == -INFINITY ? 0.f : m_new;  // nothing seen yet: every exponent is -inf
        const float corr = __builtin_amdgcn_exp2f(m - ref);
        m = m_new;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], p.scale_log2, -ref));
            sum += s[i];
        }
        l = l * corr + sum;
#pragma unroll
        for (int db = 0; db < DP / 32; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                o[db][i] *= corr;
        if (masked && lds_odd[stage] != 0u) {
            for (int x = 0; x < kTileN; ++x)
                mat.add_token(lds_v, s, o, lane, x, tb + x <= limit);
        } else {
            mat.add_values(lds_v, s, o, lane);
        }
    }

    l += __shfl_xor(l, 32);
    if (!row_ok)
        return;
    const long long row = (long long)(q0 + token) * p.Hq + head;
    if (p.num_splits > 1) {
        if (h == 0) {
            p.part_ml[row * p.num_splits + at.split] = make_float4(m, l, 1.f, 0.f);
            if (at.split == 0)  // and the parts that this prompt does not have
                for (int s = at.splits; s < p.num_splits; ++s)
                    p.part_ml[row * p.num_splits + s] = make_float4(-INFINITY, 0.f, 1.f, 0.f);
        }
        if (t0 >= t1)
            return;
        float* dst = (float*)p.part_acc + (row * p.num_splits + at.split) * p.D;
#pragma unroll
        for (int db = 0; db < DP / 32; ++db)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                const int c = 32 * db + 8 * q4 + 4 * h;
                if (c < p.D)
                    *reinterpret_cast<float4*>(dst + c) = make_float4(o[db][4 * q4], o[db][4 * q4 + 1], o[db][4 * q4 + 2], o[db][4 * q4 + 3]);
            }
        return;
    }
    const bool none = l == 0.f;
    const float inv = none ? 0.f : 1.f / l;
    if (p.lse && h == 0)
        p.lse[row] = none ? -INFINITY : m * kLn2 + logf(l);
    char* dst = (char*)p.out + row * p.D * E;
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
            const int c = 32 * db + 8 * q4 + 4 * h;
            if (c >= p.D)
                continue;
            const float x0 = o[db][4 * q4] * inv, x1 = o[db][4 * q4 + 1] * inv, x2 = o[db][4 * q4 + 2] * inv, x3 = o[db][4 * q4 + 3] * inv;
            if constexpr (E == 2)
                *reinterpret_cast<uint2*>(dst + c * 2) = make_uint2(pack_bf16(x0, x1), pack_bf16(x2, x3));
            else
                *reinterpret_cast<float4*>(dst + c * 4) = make_float4(x0, x1, x2, x3);
        }
}

// Joins the parts of a row: with states (m_i, l_i, acc_i), m = max m_i and w_i = 2^(m_i - m),
// out = sum w_i acc_i / sum w_i l_i.  LANES lanes take a row, 16 bytes of a part each; they also take its parts' (m, l, scale)
// and hand their weights round.  Bound by the partial states, all of whose loads a lane has in flight kBatch at a time.
template <typename T, bool HALF, int LANES>
__global__ __launch_bounds__(kThreads) void prompt_merge_kernel(PromptParams p)
{
    constexpr int kRowsPerBlock = kThreads / LANES, kBatch = 8, kCh = HALF ? 8 : 4;
    const int lane = threadIdx.x % LANES, first_lane = (threadIdx.x & 63) - lane, c = lane * kCh;
    const long long row = (long long)blockIdx.x * kRowsPerBlock + threadIdx.x / LANES;
    const bool row_ok = row < (long long)p.query_indptr[p.B] * p.Hq && row < p.rows;
    const int S = p.num_splits;
    const float4* ml = p.part_ml + (row_ok ? row : 0) * S;
    const char* parts = (const char*)p.part_acc + ((row_ok ? row : 0) * S * p.D + (c < p.D ? c : 0)) * (HALF ? 2 : 4);
    const long long part_bytes = (long long)p.D * (HALF ? 2 : 4);
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
                w = HALF ? u * x.y * x.z : u;
            }
        }
        const int here = min(LANES, S - s0);
        for (int k0 = 0; k0 < here; k0 += kBatch) {
            uint4 a[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k)
                a[k] = *reinterpret_cast<const uint4*>(parts + min(s0 + k0 + k, S - 1) * part_bytes);
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const float ws = __shfl(w, first_lane + min(k0 + k, LANES - 1));
                if (ws != 0.f && k0 + k < here) {  // (a part that holds nothing was not written)
                    const uint32_t v[4] = {a[k].x, a[k].y, a[k].z, a[k].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if constexpr (HALF) {
                            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&v[e]));
                            acc[2 * e] = fmaf(ws, f.x, acc[2 * e]);
                            acc[2 * e + 1] = fmaf(ws, f.y, acc[2 * e + 1]);
                        } else {
                            acc[e] = fmaf(ws, __uint_as_float(v[e]), acc[e]);
                        }
                    }
                }
            }
        }
    }
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1)
        l += __shfl_xor(l, o);
    if (!row_ok)
        return;
    const bool none = l == 0.f;
    const float inv = none ? 0.f : 1.f / l;
    if (p.lse && lane == 0)
        p.lse[row] = none ? -INFINITY : m * kLn2 + logf(l);
    if (c >= p.D)
        return;
    char* dst = (char*)p.out + (row * p.D + c) * (long long)sizeof(T);
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int e = 0; e < kCh; e += 4)
            *reinterpret_cast<uint2*>(dst + 2 * e) =
                make_uint2(pack_bf16(acc[e] * inv, acc[e + 1] * inv), pack_bf16(acc[e + 2] * inv, acc[e + 3] * inv));
    } else {
        *reinterpret_cast<float4*>(dst) = make_float4(acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
    }
}

template <typename T, bool HALF, int LANES> void launch_merge(const PromptParams& p, hipStream_t s)
{
    constexpr int kRowsPerBlock = kThreads / LANES;
    hipLaunchKernelGGL((prompt_merge_kernel<T, HALF, LANES>), dim3((unsigned)((p.rows + kRowsPerBlock - 1) / kRowsPerBlock)),
                       dim3(kThreads), 0, s, p);
}

template <typename T>
hipError_t launch(const PromptParams& p, hipStream_t s)
{
    const dim3 grid((unsigned)((long long)p.tiles * p.num_splits * p.Hkv)), block(kThreads);
    if (sizeof(T) == 2 && (p.D == 64 || p.D == 128)) {
        const hipError_t e = launch_prompt_mfma(p, s);
        if (e != hipSuccess)
            return e;
        if (p.num_splits > 1)
            p.D == 64 ? launch_merge<T, true, 8>(p, s) : launch_merge<T, true, 16>(p, s);
        return hipGetLastError();
    }
    if (p.D <= 64) {
        hipLaunchKernelGGL((prompt_attn_kernel<T, 64>), grid, block, 0, s, p);
        if (p.num_splits > 1)
            launch_merge<T, false, 16>(p, s);
    } else if (p.D <= 128) {
        hipLaunchKernelGGL((prompt_attn_kernel<T, 128>), grid, block, 0, s, p);
        if (p.num_splits > 1)
            launch_merge<T, false, 32>(p, s);
    } else {
        hipLaunchKernelGGL((prompt_attn_kernel<T, 256>), grid, block, 0, s, p);
        if (p.num_splits > 1)
            launch_merge<T, false, 64>(p, s);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_prompt_attn(const PromptParams& p, hipStream_t s)
{
    return p.dtype == 1 ? launch<__bf16>(p, s) : launch<float>(p, s);
}

}  // namespace spd
