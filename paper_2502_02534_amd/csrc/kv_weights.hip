// How much of the queries' attention every cached token got:
//   w'[b, j, t] = decay w[b, j, t] + sum over the query rows (i, h) that see t of 2^(scale_log2 q . k_t - lse_log2) f
// f, next to 1, takes back what lse_log2 = lse log2(e) loses by its rounding to 24 bits: one error for all of a row's tokens, 5e-7 of them at an lse
// of 10.  The sums multiply by it as they add.  The scale's own rounding, up to 6e-8 of a score, is taken back where few rows wait for memory; beside
// many rows' products the instruction for it would cost 7 to 12 %.
//
// Rows are the (query, head of the group) pairs of a KV head.  The products are taken transposed, S^T = K Q^T: a lane of the
// accumulator has one row's scores of several tokens, so the row's log-sum-exp is one number a lane, and a token's sum over
// the rows stays in its register until the end, when the lanes' shares are added.  A weight has one owner (or one for each
// part of the rows, which a second launch adds in order), so no sum depends on who comes first.
//
//   few rows (up to 32: one step's queries over a sample's own tokens): a wavefront keeps the rows' fragments in registers and streams
//     the keys: whole lines, marked as used once, the next tile's under way while it works on this one, which goes through LDS of the
//     wavefront's own to the lanes that multiply it.  Bound: HBM, K read once (1024 samples of up to 2048 paged tokens, 8 heads of 128
//     channels, 2.2 GB: 376 us, 5.9 TB/s; loads in the products' order 449 where these took 387).
//   many rows (samples over their shared prompt, a prompt over itself): a wavefront keeps 64 tokens' keys in registers (32 in fp32), and
//     the rows pass by in blocks of 32 through LDS, shared by a workgroup's four wavefronts; in bf16 the exponentials of one half of the
//     tokens run between the products of the other.  Bound: matrix pipe and vector ALU together, and the clock that their power leaves:
//     a block takes 16 products of 32 clocks beside 32 exponentials and 64 fma a lane (128 channels).  16384 tokens of 64 / 8 heads
//     2.22 ms: 1.0 PFLOP/s of the products that the rows need, matrix pipe 56 % busy, 1.83 GHz; 4096 fp32 tokens of 16 / 4 heads of 64
//     channels 172 us (100 TFLOP/s).
//     Causal: the last rows, which every tile sees, come first, and first tiles, which see most, are launched first.  Rows in eight parts
//     instead of one, which even out the tiles' work: 2.65 -> 2.28 ms; parts of the same rows for every tile, which keep them in the L2
//     (7.5 GB fetched otherwise), win 3 % there and lose 5 to 70 % on shorter prompts, whose parts are then half empty.
//     64 samples over a prompt of 8192, 32 / 8 heads: 11.1 us, latency (a chain of loads, eight blocks, the sums over the lanes).  All rows in
//     LDS at once, and wavefronts that walk several tiles without a barrier: 12.4, and 80 against 84 for 8 x 64 queries over 1k to 16k tokens.
#include "prompt_plan.h"
#include "spd_internal.h"

#include <type_traits>

namespace spd {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float floatx4;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float floatx16;

constexpr int kWaves = 4;
// Wavefronts of a workgroup where each works by itself.  Where pages lie anywhere, workgroups of one spread the heads of a page over the chip:
// 1024 samples of up to 2048 paged tokens, 8 heads of 128 channels, 1 / 2 / 4 / 8 of them 376 / 378 / 380 / 388 us, 64 samples 26.7 / 28.3 / 30.4 / 30.5
// (contiguous, 1024 of up to 1024 tokens: 200 / 191 / 188 / 195).
constexpr int few_waves(bool paged) { return paged ? 1 : 4; }

__device__ __forceinline__ bf16x8 as_bf16x8(const uint4& v) { return *reinterpret_cast<const bf16x8*>(&v); }
__device__ __forceinline__ float part_of(const uint4& v, int e)
{
    return __uint_as_float(e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w);
}

// What a row's lse does to its terms: an exponent, -lse in base 2, and the factor that its rounding needs.  A row that is not there, or saw
// nothing, has -inf: it adds 2^-inf = 0.
struct Shift {
    float below = -INFINITY, by = 1.f;
};
__device__ __forceinline__ Shift shift_of(float lse, bool there)
{
    constexpr float kLog2eRest = 1.92596299e-8f;  // log2(e) - kLog2e
    const float x = lse * kLog2e, lost = __builtin_fmaf(lse, kLog2eRest, __builtin_fmaf(lse, kLog2e, -x));
    Shift s;
    s.below = !there || lse == -INFINITY ? -INFINITY : -x;
    // (an lse of 2^23 and more has no last place that means anything, and an infinite one loses NaN)
    s.by = __builtin_amdgcn_fmed3f(__builtin_fmaf(lost, -kLn2, 1.f), 0.5f, 2.f);
    return s;
}

// Sum over the 16 lanes of a lane row.
template <int CTRL> __device__ __forceinline__ float add_dpp(float v)
{
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float over_row(float v)
{
    return add_dpp<0x121>(add_dpp<0x122>(add_dpp<0x124>(add_dpp<0x128>(v))));  // rotations by 8, 4, 2, 1
}

// 16-byte piece `piece` of token t's key, KV head j; `head_pieces` of them, zeros behind.
template <bool PAGED> struct Keys {
    const uint4* base;
    const int* pages;
    long long head_at, token_pieces, page_pieces;
    __device__ __forceinline__ Keys(const KvWeightsParams& p, int b, int j, int head_pieces)
    {
        const int first = p.kv_indptr[b];
        const int per = p.dtype == 1 ? 8 : 4;
        if (PAGED) {
            base = (const uint4*)p.k;
            pages = p.pages + first;
            token_pieces = head_pieces;
            page_pieces = (long long)p.Hkv * 16 * head_pieces;
            head_at = (long long)j * 16 * head_pieces;
        } else {
            token_pieces = p.kv_stride / per;
            base = (const uint4*)p.k + (long long)first * token_pieces;
            pages = nullptr;
            page_pieces = 0;
            head_at = (long long)j * head_pieces;
        }
    }
    __device__ __forceinline__ const uint4* row(int t) const
    {
        return PAGED ? base + (long long)pages[t >> 4] * page_pieces + head_at + (t & 15) * token_pieces : base + head_at + (long long)t * token_pieces;
    }
};

// ---- few rows: the keys stream by --------------------------------------------------------------------------------

// bf16: 16 x 16 x 32 products, step s takes pieces 4 s + g of a row (g = lane / 16); fp32: 16 x 16 x 4, piece 4 s + g's four elements
// one after another.  Either way a lane's operand is 16-byte pieces of its row.
template <bool BF16> __device__ __forceinline__ floatx4 product16(const uint4& k, const uint4& q, floatx4 c)
{
    if constexpr (BF16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(k), as_bf16x8(q), c, 0, 0, 0);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(part_of(k, e), part_of(q, e), c, 0, 0, 0);
        return c;
    }
}

// P: 16-byte pieces of a padded head (D = 64, 128, 256 in bf16: 8, 16, 32); SUB: 16-token halves of a tile; NB: blocks of 16 rows; ONE: a stretch
// is one tile: no second one's registers (20 sequences of up to 640 tokens, 8 heads of 256 channels 8.5 -> 7.0 us).
template <bool BF16, int P, int SUB, int NB, bool PAGED, bool ONE>
__global__ __launch_bounds__(few_waves(PAGED) * 64) void kv_weights_few(KvWeightsParams p, int chunk, int chunks)
{
    constexpr int kSteps = P / 4, kTile = 16 * SUB, kLoads = kTile * P / 64, kPitch = P + 1, kFewWaves = few_waves(PAGED);  // (a piece between rows: bank conflicts)
    __shared__ uint4 lds[kFewWaves][kTile * kPitch];
    const int lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
    const int item = __builtin_amdgcn_readfirstlane(blockIdx.x * kFewWaves + (threadIdx.x >> 6));
    // KV head fastest: the heads of a token lie beside each other.  The later a stretch, the fewer sequences have it: each starts three sequences on, or a
    // CU would get the long ones again and again (64 paged sequences of up to 2048 tokens 29.3 us, so 26.7; 512 189.8 and 187.4)
    const int j = item % p.Hkv, rest = item / p.Hkv, at = rest / p.B;
    int b = rest - at * p.B + 3 * at;
    if (b >= p.B)
        b = b < 2 * p.B ? b - p.B : b % p.B;
    if (at >= chunks)
        return;
    const int L = min(p.kv_lens[b], p.max_kv), t0 = at * chunk, t1 = min(L, t0 + chunk);
    if (t0 >= t1)
        return;
    const int q0 = p.query_indptr[b], n = max(min(p.query_indptr[b + 1] - q0, p.max_query), 0), rows = n * p.G;
    const int head_pieces = p.D / (BF16 ? 8 : 4);
    const Keys<PAGED> keys(p, b, j, head_pieces);

    uint4 q[NB][kSteps];
    Shift shift[NB];  // of the lane's row
    int limit[NB];    // last token that it sees
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int r = nb * 16 + col, i = min(r, max(rows - 1, 0)) / p.G, h = j * p.G + min(r, max(rows - 1, 0)) % p.G;
        const bool there = r < rows;
        shift[nb] = shift_of(there ? p.lse[(long long)(q0 + i) * p.Hq + h] : 0.f, there);
        limit[nb] = !there ? -1 : p.causal ? L - n + i : L;
        const uint4* const from = (const uint4*)p.q + (long long)(q0 + i) * (p.q_stride / (BF16 ? 8 : 4)) + (long long)h * head_pieces;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            q[nb][s] = make_uint4(0u, 0u, 0u, 0u);
            if (there && 4 * s + g < head_pieces)
                q[nb][s] = from[4 * s + g];
        }
    }
    // the lanes that store: 4 SUB of each lane row, token 16 (col / 4) + 4 g + col % 4 of the tile
    const int mine = 16 * (col >> 2) + 4 * g + (col & 3);
    const bool stores = col < 4 * SUB;
    const long long out_at = ((long long)b * p.Hkv + j) * p.stride;
    // A tile's rows are loaded as they lie, P pieces one after another (whole lines, used once), and get to the lanes that multiply them
    // through LDS of the wavefront's own.
    uint4* const mine_lds = lds[threadIdx.x >> 6];
    const int in_row = lane % P, in_tile = lane / P;  // piece and first row of a lane's loads
    const bool has_piece = in_row < head_pieces;
    // (tiles start with a page; its number is fetched a tile ahead of its rows, beside loads into lanes: a scalar would be waited for at once)
    const int last_page = (t1 - 1) >> 4;
    int next_page[SUB], any_lane = 0;
    asm("" : "+v"(any_lane));
    const auto fetch_pages = [&](int tb, int lane_zero) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < SUB; ++u)
            next_page[u] = PAGED ? keys.pages[min((tb >> 4) + u, last_page) + lane_zero] : 0;
    };
    const auto load = [&](int tb, uint4 (&k)[kLoads], float& old) __attribute__((always_inline)) {
        typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
        int page[SUB];
#pragma unroll
        for (int u = 0; u < SUB; ++u)
            page[u] = next_page[u];
        if (!ONE)
            fetch_pages(tb + kTile, any_lane);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int t = min(tb + i * (64 / P) + in_tile, t1 - 1);
            const uint4* const row = PAGED ? keys.base + page[i * (64 / P) / 16] * keys.page_pieces + keys.head_at + (t & 15) * keys.token_pieces
                                           : keys.row(t);
            const u32x4 v = __builtin_nontemporal_load((const u32x4*)(row + (has_piece ? in_row : 0)));
            k[i] = make_uint4(v[0], v[1], v[2], v[3]);
        }
        old = 0.f;
        if (p.weights)
            old = p.weights[out_at + min(tb + mine, t1 - 1)];
    };
    const auto work = [&](int tb, const uint4 (&loaded)[kLoads], float old) __attribute__((always_inline)) {
        float total = 0.f;
        wave_sync();
        if (has_piece) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                mine_lds[(i * (64 / P) + in_tile) * kPitch + in_row] = loaded[i];
        }
        wave_sync();
        uint4 k[SUB][kSteps];
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int s = 0; s < kSteps; ++s)
                k[u][s] = mine_lds[(16 * u + col) * kPitch + 4 * s + g];
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            floatx4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                floatx4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < kSteps; ++s)
                    c = product16<BF16>(k[u][s], q[nb][s], c);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    // (an infinite score stays what it is)
                    const float rest = __builtin_amdgcn_fmed3f(c[i], -3.402823466e38f, 3.402823466e38f) * p.scale_rest;
                    const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(c[i], p.scale_log2, shift[nb].below) + rest);
                    sum[i] = __builtin_fmaf(tb + 16 * u + 4 * g + i <= limit[nb] ? x : 0.f, shift[nb].by, sum[i]);  // (a row that is not there sees nothing)
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float all = over_row(sum[i]);
                total = col == 4 * u + i ? all : total;
            }
        }
        total = p.weights ? __builtin_fmaf(p.decay, old, total) : total;
        if (stores && tb + mine < t1)
            p.weights_out[out_at + tb + mine] = total;
    };
    if (!has_piece) {  // (zeros behind a head's channels, once)
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            mine_lds[(i * (64 / P) + in_tile) * kPitch + in_row] = make_uint4(0u, 0u, 0u, 0u);
    }
    uint4 ka[kLoads], kb[kLoads];
    float oa, ob;
    fetch_pages(t0, 0);
    load(t0, ka, oa);
    if constexpr (ONE) {
        work(t0, ka, oa);
        return;
    }
    // (no branch around a load in the loop: after one, all loads that may be under way would be waited for)
    int tb = t0;
    for (; tb + 2 * kTile < t1; tb += 2 * kTile) {
        load(tb + kTile, kb, ob);
        work(tb, ka, oa);
        load(tb + 2 * kTile, ka, oa);
        work(tb + kTile, kb, ob);
    }
    if (tb + kTile < t1) {
        load(tb + kTile, kb, ob);
        work(tb, ka, oa);
        work(tb + kTile, kb, ob);
    } else {
        work(tb, ka, oa);
    }
}

// ---- many rows -----------------------------------------------------------------------------------------------------

// What a workgroup of the other kernels takes: `tokens` keys from t0 on of KV head j of sequence b, and the row blocks
// first .. last - 1 of 32 rows that see any of them.
struct Unit {
    bool any;
    int b, j, t0, L, q0, n, rows, first, last, split;
};

__device__ __forceinline__ Unit find_unit(const KvWeightsParams& p, int tokens)
{
    Unit u;
    const int j = blockIdx.x % p.Hkv;
    const int rest = blockIdx.x / p.Hkv;
    // causal tiles see the fewer rows the later they are: first tiles first
    const int tile = rest / (p.B * p.splits), rem = rest % (p.B * p.splits);
    u.j = j;
    u.b = rem / p.splits;
    u.split = rem % p.splits;
    u.t0 = tile * tokens;
    u.L = min(p.kv_lens[u.b], p.max_kv);
    u.any = u.t0 < u.L;
    if (!u.any)
        return u;
    u.q0 = p.query_indptr[u.b];
    u.n = max(min(p.query_indptr[u.b + 1] - u.q0, p.max_query), 0);
    u.rows = u.n * p.G;
    const int hidden = p.causal ? min(max(u.t0 - (u.L - u.n), 0), u.n) * p.G : 0;  // rows that see nothing of the tile
    const int lo = hidden / 32, hi = (u.rows + 31) / 32, per = (hi - lo + p.splits - 1) / p.splits;
    u.first = lo + min(u.split * per, hi - lo);
    u.last = min(u.first + per, hi);
    return u;
}

// Sums of V values over the 32 lanes of a half: value c of the half's lane c afterwards (V = 16: lanes c and c + 16 alike).
template <int V> __device__ __forceinline__ float over_columns(float (&v)[V])
{
    const int lane = threadIdx.x & 63;
    int kept = V;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        if (V == 16 && o == 16) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                v[i] += __shfl_xor(v[i], 16);
            continue;
        }
        kept >>= 1;
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            if (i < kept) {
                const bool up = (lane & o) != 0;
                const float lo = v[i] + 0.f, hi = v[i + kept] + 0.f;  // (values: a choice of places would be one of addresses)
                v[i] = (up ? hi : lo) + __shfl_xor(up ? lo : hi, o);
            }
        }
    }
    return v[0];
}

// The unit's weights: value c of half h is token 32 (c / 16) + 8 (c % 16 / 4) + 4 h + c % 4 of the wavefront's.
template <int V> __device__ __forceinline__ void store(const KvWeightsParams& p, const Unit& u, int tw, float (&v)[V])
{
    const int lane = threadIdx.x & 63, c = lane & (V - 1), h = lane >> 5;
    const float total = over_columns(v);
    const int t = tw + 32 * (c >> 4) + 8 * ((c & 15) >> 2) + 4 * h + (c & 3);
    if (t >= u.L || (lane & 31) >= V)
        return;
    if (p.splits > 1) {
        p.part[(((long long)u.split * p.B + u.b) * p.Hkv + u.j) * p.max_kv + t] = total;
        return;
    }
    const long long at = ((long long)u.b * p.Hkv + u.j) * p.stride + t;
    p.weights_out[at] = p.weights ? __builtin_fmaf(p.decay, p.weights[at], total) : total;
}

// bf16.  D: channels of a padded head.  A row in LDS is 16 bytes longer than its channels, so that sixteen rows' equal pieces take all 64 banks.
template <int D> struct Shape {
    static constexpr int kRow = 2 * D + 16, kBlock = 32 * kRow, kPieces = D / 8, kSteps = D / 16;
    static constexpr int kCopyRows = kWaves * 64 / kPieces, kCopies = 32 / kCopyRows;
};

constexpr int kManyTokens = 64;  // of a wavefront

// A wavefront's tokens are two halves of 32.  While the products of one half's scores with a block of rows run, the other half's scores
// (of the same block, or the one before) become weights, an element every few clocks of the matrix pipe; the rows' fragments
// stay in registers for both halves, and the next block's take their place behind the last product that reads them.
template <int D, bool FULL, bool EVEN>  // FULL: the heads have D channels, not fewer; EVEN: the group divides 32
__global__ __launch_bounds__(kWaves * 64, D <= 128 ? 2 : 1) void kv_weights_many(KvWeightsParams p)
{
    using S = Shape<D>;
    __shared__ __align__(16) char lds[2 * S::kBlock];
    const Unit u = find_unit(p, kWaves * kManyTokens);
    if (!u.any)
        return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, h = lane >> 5;
    const int tw = u.t0 + wave * kManyTokens, head_pieces = FULL ? S::kPieces : p.D / 8, G = p.G;
    float sums[32];
#pragma unroll
    for (int i = 0; i < 32; ++i)
        sums[i] = 0.f;
    if (u.first < u.last) {
        // ---- rows, the last block first: from memory into registers two blocks ahead, into LDS one ahead.  A thread copies the same
        // 16-byte piece of the same rows of every block.  Rows behind the last one repeat its query; nothing is added for them.
        const long long q_bytes = p.q_stride * 2;
        const int piece = tid % S::kPieces, copy_row = tid / S::kPieces, head_bytes = head_pieces * 16;
        const bool has_piece = FULL || piece < head_pieces;
        const char* const q_seq = (const char*)p.q + (long long)u.q0 * q_bytes + (long long)u.j * G * head_bytes;
        const float* const lse_seq = p.lse + (long long)u.q0 * p.Hq + (long long)u.j * G;
        const int piece_at = has_piece ? piece * 16 : 0;
        uint4 staged[S::kCopies];
        const auto copy_any = [&](int block, int c) __attribute__((always_inline)) {  // of any block
            const int r = block * 32 + c * S::kCopyRows + copy_row;
            return *(const uint4*)(q_seq + min(r / G, u.n - 1) * q_bytes + r % G * head_bytes + piece_at);
        };
        const auto lse_any = [&](int block) __attribute__((always_inline)) {
            const int r = block * 32 + col;
            return lse_seq[(long long)min(r / G, u.n - 1) * p.Hq + r % G];
        };
        // EVEN: a whole block's rows lie as block 0's do, 32 / G queries a block apart (a sequence of less than a block has no other)
        unsigned copy_at[S::kCopies], lse_off = 0;
        if (EVEN) {
#pragma unroll
            for (int c = 0; c < S::kCopies; ++c) {
                const int r = c * S::kCopyRows + copy_row;
                copy_at[c] = (unsigned)(min(r / G, u.n - 1) * q_bytes + r % G * head_bytes + piece_at);
            }
            lse_off = (unsigned)(min(col / G, u.n - 1) * p.Hq + col % G) * 4u;
        }
        const int block_queries = 32 / G;
        int fetched = u.last - 1;
        float lse_next = lse_any(fetched);
#pragma unroll
        for (int c = 0; c < S::kCopies; ++c)
            staged[c] = copy_any(fetched, c);
        const auto fetch = [&]() __attribute__((always_inline)) {  // the block before (block 0's where there is none: not used)
            fetched = fetched > u.first ? fetched - 1 : 0;
            if (EVEN) {
                const char* const from = q_seq + (long long)fetched * block_queries * q_bytes;
#pragma unroll
                for (int c = 0; c < S::kCopies; ++c)
                    staged[c] = *(const uint4*)(from + copy_at[c]);
            } else {
#pragma unroll
                for (int c = 0; c < S::kCopies; ++c)
                    staged[c] = copy_any(fetched, c);
            }
        };
        int lse_block = fetched;
        const auto fetch_lse = [&]() __attribute__((always_inline)) {
            lse_block = lse_block > u.first ? lse_block - 1 : 0;
            if (EVEN)
                lse_next = *(const float*)((const char*)(lse_seq + (long long)lse_block * block_queries * p.Hq) + lse_off);
            else
                lse_next = lse_any(lse_block);
        };
        char* const lds_put = lds + copy_row * S::kRow + piece * 16;
        const auto put = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
            for (int c = 0; c < S::kCopies; ++c) {
                const uint4 v = staged[c];
                *(uint4*)(lds_put + slot * S::kBlock + c * S::kCopyRows * S::kRow) =
                    FULL ? v : make_uint4(has_piece ? v.x : 0u, has_piece ? v.y : 0u, has_piece ? v.z : 0u, has_piece ? v.w : 0u);
            }
        };
        // ---- keys: A operand, row = token, channels 16 s + 8 h (tokens past the end repeat the last one)
        uint4 k[2][S::kSteps];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int t = min(tw + 32 * x + col, u.L - 1);
            const uint4* const row = p.page_size ? Keys<true>(p, u.b, u.j, head_pieces).row(t) : Keys<false>(p, u.b, u.j, head_pieces).row(t);
#pragma unroll
            for (int s = 0; s < S::kSteps; ++s) {
                k[x][s] = make_uint4(0u, 0u, 0u, 0u);
                if (FULL || 2 * s + h < head_pieces)
                    k[x][s] = row[2 * s + h];
            }
        }
        put(0);
        fetch();
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        uint4 f[S::kSteps];
        const char* const lds_row = lds + col * S::kRow + h * 16;
#pragma unroll
        for (int s = 0; s < S::kSteps; ++s)
            f[s] = *(const uint4*)(lds_row + 32 * s);
        floatx16 sc[2];
#pragma unroll
        for (int e = 0; e < 16; ++e)
            sc[1][e] = 0.f;
        Shift shift_was, shift;
        float lse = 0.f;
        int limit_was = 0, limit = 0;
        const int hide = u.L - u.n;
        // scores of half x become weights, element by element: exponent of e, exponential of e - 1, sum of e - 2
        float ex[16];
        const auto soft = [&](auto mask_tag, int x, int e, const Shift& b, int lim) __attribute__((always_inline)) {
            constexpr bool MASK = decltype(mask_tag)::value;
            if (e < 16)
                ex[e] = __builtin_fmaf(sc[x][e], p.scale_log2, b.below);
            if (e >= 1 && e < 17)
                ex[e - 1] = __builtin_amdgcn_exp2f(ex[e - 1]);
            if (e >= 2 && e < 18) {
                const int d = e - 2;
                float w = ex[d];
                if (MASK)
                    w = tw + 32 * x + (d & 3) + 8 * (d >> 2) + 4 * h <= lim ? w : 0.f;
                sums[16 * x + d] = __builtin_fmaf(w, b.by, sums[16 * x + d]);
            }
        };
        const auto phase = [&](auto x_tag, auto mask_tag, int slot, const Shift& b, int lim, auto beside) __attribute__((always_inline)) {
            constexpr int X = decltype(x_tag)::value;
#pragma unroll
            for (int e = 0; e < 16; ++e)
                sc[X][e] = 0.f;
#pragma unroll
            for (int s = 0; s < S::kSteps; ++s) {
                sc[X] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(k[X][s]), as_bf16x8(f[s]), sc[X], 0, 0, 0);
                if (X == 1)
                    f[s] = *(const uint4*)(lds_row + slot * S::kBlock + 32 * s);
                // (beside the first product the other half's last one still runs)
                if (s == 0) {
                    __builtin_amdgcn_sched_barrier(0);
                    beside();
                } else
#pragma unroll
                    for (int e = (s - 1) * 18 / (S::kSteps - 1); e < s * 18 / (S::kSteps - 1); ++e)
                        soft(mask_tag, 1 - X, e, b, lim);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        const std::integral_constant<int, 0> lower{};
        const std::integral_constant<int, 1> upper{};
        const auto block = [&](auto mask_tag, int slot) __attribute__((always_inline)) {
            // the next block's rows go to LDS, and the loads of the one after start
            phase(lower, mask_tag, slot, shift_was, limit_was, [&]() __attribute__((always_inline)) {
                lse = lse_next;
                put(slot);
                fetch_lse();
                fetch();
            });
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            phase(upper, mask_tag, slot, shift, limit, [&]() __attribute__((always_inline)) { shift = shift_of(lse, true); });
            shift_was = shift;
        };
        // blocks of which every row sees all of this wavefront's tokens
        const int whole_first = p.causal ? (max(tw + kManyTokens - 1 - hide, 0) * G + 31) / 32 : 0, whole_last = u.rows / 32;
        int slot = 1, at = u.last - 1;
#pragma unroll 1
        while (at >= u.first) {  // (a loop of its own for either kind)
#pragma unroll 1
            for (; at >= u.first && (at < whole_first || at + 1 >= whole_last); --at) {
                const int r = at * 32 + col;
                limit = r >= u.rows ? -1 : p.causal ? hide + r / G : u.L;
                limit_was = r + 32 >= u.rows ? -1 : p.causal ? hide + (r + 32) / G : u.L;
                block(std::true_type{}, slot);
                slot ^= 1;
            }
#pragma unroll 1
            for (; at >= u.first && at >= whole_first && at + 1 < whole_last; --at) {
                block(std::false_type{}, slot);
                slot ^= 1;
            }
        }
        const int r = u.first * 32 + col;
        limit = r >= u.rows ? -1 : p.causal ? hide + r / G : u.L;
#pragma unroll
        for (int e = 0; e < 18; ++e)
            soft(std::true_type{}, 1, e, shift, limit);
    }
    store<32>(p, u, tw, sums);
}

// fp32: 32 tokens a wavefront; the rows go through LDS as in bf16, a block ahead (a product of fp32 takes 16 times as long).
// P: 16-byte pieces of a padded head.
template <int P>
__global__ __launch_bounds__(kWaves * 64, P <= 32 ? 2 : 1) void kv_weights_many_f32(KvWeightsParams p)
{
    constexpr int kSteps = P / 2, kPitch = P + 1, kCopies = 32 * P / (kWaves * 64);
    static_assert(32 * P % (kWaves * 64) == 0 && P % 2 == 0, "whole copies, and rows that end in another bank");
    __shared__ uint4 lds[2][32 * kPitch];
    const Unit u = find_unit(p, kWaves * 32);
    if (!u.any)
        return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, h = lane >> 5;
    const int tw = u.t0 + wave * 32, head_pieces = p.D / 4, G = p.G;
    float sums[16];
#pragma unroll
    for (int i = 0; i < 16; ++i)
        sums[i] = 0.f;
    if (u.first < u.last) {
        const uint4* const q_seq = (const uint4*)p.q + (long long)u.q0 * (p.q_stride / 4) + (long long)u.j * G * head_pieces;
        uint4 staged[kCopies];
        const auto fetch = [&](int at) __attribute__((always_inline)) {
#pragma unroll
            for (int c = 0; c < kCopies; ++c) {
                const int x = c * kWaves * 64 + tid, r = min(at * 32 + x / P, u.rows - 1), piece = x % P;
                staged[c] = make_uint4(0u, 0u, 0u, 0u);
                if (piece < head_pieces)
                    staged[c] = q_seq[r / G * (p.q_stride / 4) + r % G * head_pieces + piece];
            }
        };
        const auto put = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
            for (int c = 0; c < kCopies; ++c) {
                const int x = c * kWaves * 64 + tid;
                lds[slot][x / P * kPitch + x % P] = staged[c];
            }
        };
        float lse;
        int query;
        const auto fetch_lse = [&](int at) __attribute__((always_inline)) {
            const int r = min(at * 32 + col, u.rows - 1);
            query = r / G;
            lse = p.lse[(long long)(u.q0 + query) * p.Hq + u.j * G + r % G];
        };
        fetch(u.last - 1);
        fetch_lse(u.last - 1);
        uint4 k[kSteps];
        const int tk = min(tw + col, u.L - 1);
        const uint4* const row = p.page_size ? Keys<true>(p, u.b, u.j, head_pieces).row(tk) : Keys<false>(p, u.b, u.j, head_pieces).row(tk);
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            k[s] = make_uint4(0u, 0u, 0u, 0u);
            if (2 * s + h < head_pieces)
                k[s] = row[2 * s + h];
        }
        put(0);
        // (causal: blocks that see none of this wavefront's tokens are only copied)
        const int first = tw >= u.L ? u.last : p.causal ? min(max(tw - (u.L - u.n), 0), u.n) * G / 32 : 0;
        int slot = 0;
#pragma unroll 1
        for (int at = u.last - 1; at >= u.first; --at) {
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            const bool there = at * 32 + col < u.rows;
            const Shift shift = shift_of(lse, there);
            const int limit = !there ? -1 : p.causal ? u.L - u.n + query : u.L;
            if (at > u.first) {
                fetch(at - 1);
                fetch_lse(at - 1);
            }
            if (at >= first) {
                floatx16 c;
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    c[e] = 0.f;
                const uint4* const from = &lds[slot][col * kPitch + h];
#pragma unroll
                for (int s = 0; s < kSteps; ++s) {
                    const uint4 f = from[2 * s];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        c = __builtin_amdgcn_mfma_f32_32x32x2f32(part_of(k[s], e), part_of(f, e), c, 0, 0, 0);
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(c[e], p.scale_log2, shift.below));
                    sums[e] = __builtin_fmaf(tw + (e & 3) + 8 * (e >> 2) + 4 * h <= limit ? w : 0.f, shift.by, sums[e]);
                }
            }
            slot ^= 1;
            if (at > u.first)
                put(slot);
        }
    }
    store<16>(p, u, tw, sums);
}

// Adds the parts of the rows in order.
__global__ __launch_bounds__(256) void kv_weights_join(KvWeightsParams p)
{
    const int t = blockIdx.x * 256 + threadIdx.x, bj = blockIdx.y, b = bj / p.Hkv;
    if (t >= min(p.kv_lens[b], p.max_kv))
        return;
    const long long at = (long long)bj * p.stride + t, pitch = (long long)p.B * p.Hkv * p.max_kv;
    const float old = p.weights ? p.weights[at] : 0.f;
    const float* const part = p.part + (long long)bj * p.max_kv + t;
    float total = 0.f;
    for (int s0 = 0; s0 < p.splits; s0 += 8) {  // (eight loads under way)
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            x[i] = part[min(s0 + i, p.splits - 1) * pitch];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            total += s0 + i < p.splits ? x[i] : 0.f;
    }
    p.weights_out[at] = p.weights ? __builtin_fmaf(p.decay, old, total) : total;
}

template <bool BF16, int P, int SUB, int NB> void few(const KvWeightsParams& p, hipStream_t s)
{
    // a wavefront's stretch of tokens: long ones keep its loads going, short ones fill the card
    const long long pairs = (long long)p.B * p.Hkv;
    int chunk = 256;
    while (chunk > 16 * SUB && pairs * ((p.max_kv + chunk - 1) / chunk) < 4096)
        chunk /= 2;
    const int chunks = (p.max_kv + chunk - 1) / chunk;
    const int waves = few_waves(p.page_size != 0);
    const dim3 grid((unsigned)((pairs * chunks + waves - 1) / waves)), block(waves * 64);
    const bool one = chunk == 16 * SUB;
    if (p.page_size && one)
        hipLaunchKernelGGL((kv_weights_few<BF16, P, SUB, NB, true, true>), grid, block, 0, s, p, chunk, chunks);
    else if (p.page_size)
        hipLaunchKernelGGL((kv_weights_few<BF16, P, SUB, NB, true, false>), grid, block, 0, s, p, chunk, chunks);
    else if (one)
        hipLaunchKernelGGL((kv_weights_few<BF16, P, SUB, NB, false, true>), grid, block, 0, s, p, chunk, chunks);
    else
        hipLaunchKernelGGL((kv_weights_few<BF16, P, SUB, NB, false, false>), grid, block, 0, s, p, chunk, chunks);
}

}  // namespace

hipError_t launch_kv_weights(const KvWeightsParams& p, hipStream_t s)
{
    const bool bf16 = p.dtype == 1;
    const long long rows = (long long)p.max_query * p.G;
    if (rows <= plan::kWeightsFewRows) {
        const int pieces = p.D / (bf16 ? 8 : 4);
        if (bf16) {
            if (rows <= 16)
                pieces <= 8 ? few<true, 8, 2, 1>(p, s) : pieces <= 16 ? few<true, 16, 2, 1>(p, s) : few<true, 32, 1, 1>(p, s);
            else
                pieces <= 8 ? few<true, 8, 2, 2>(p, s) : pieces <= 16 ? few<true, 16, 2, 2>(p, s) : few<true, 32, 1, 2>(p, s);
        } else {
            if (rows <= 16)
                pieces <= 16 ? few<false, 16, 1, 1>(p, s) : pieces <= 32 ? few<false, 32, 1, 1>(p, s) : few<false, 64, 1, 1>(p, s);
            else
                pieces <= 16 ? few<false, 16, 1, 2>(p, s) : pieces <= 32 ? few<false, 32, 1, 2>(p, s) : few<false, 64, 1, 2>(p, s);
        }
        return hipGetLastError();
    }
    const int tokens = plan::weights_tile_tokens(bf16), tiles = (p.max_kv + tokens - 1) / tokens;
    const long long units = (long long)tiles * p.B * p.splits;
    const dim3 grid((unsigned)(units * p.Hkv)), block(kWaves * 64);
    const bool even = 32 % p.G == 0;
#define SPD_MANY_BF16(W) \
    if (p.D == W && even) \
        hipLaunchKernelGGL((kv_weights_many<W, true, true>), grid, block, 0, s, p); \
    else if (p.D == W) \
        hipLaunchKernelGGL((kv_weights_many<W, true, false>), grid, block, 0, s, p); \
    else if (even) \
        hipLaunchKernelGGL((kv_weights_many<W, false, true>), grid, block, 0, s, p); \
    else \
        hipLaunchKernelGGL((kv_weights_many<W, false, false>), grid, block, 0, s, p)
    if (bf16) {
        if (p.D <= 64) {
            SPD_MANY_BF16(64);
        } else if (p.D <= 128) {
            SPD_MANY_BF16(128);
        } else {
            SPD_MANY_BF16(256);
        }
    } else {
        if (p.D <= 64) {
            hipLaunchKernelGGL(kv_weights_many_f32<16>, grid, block, 0, s, p);
        } else if (p.D <= 96) {
            hipLaunchKernelGGL(kv_weights_many_f32<24>, grid, block, 0, s, p);
        } else if (p.D <= 128) {
            hipLaunchKernelGGL(kv_weights_many_f32<32>, grid, block, 0, s, p);
        } else if (p.D <= 192) {
            hipLaunchKernelGGL(kv_weights_many_f32<48>, grid, block, 0, s, p);
        } else {
            hipLaunchKernelGGL(kv_weights_many_f32<64>, grid, block, 0, s, p);
        }
    }
#undef SPD_MANY_BF16
    hipError_t rc = hipGetLastError();
    if (rc == hipSuccess && p.splits > 1) {
        hipLaunchKernelGGL(kv_weights_join, dim3((p.max_kv + 255) / 256, p.B * p.Hkv), dim3(256), 0, s, p);
        rc = hipGetLastError();
    }
    return rc;
}

}  // namespace spd
