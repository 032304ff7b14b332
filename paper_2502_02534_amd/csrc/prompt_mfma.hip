// prompt_attn for bf16: the tiled kernel (prompt_attn.hip holds that for fp32 and the definition of rows and parts).
// Heads of 64, 128 and 256 channels fill a tile's rows; other dimensions run in the next larger of these, their missing
// channels zeros that are put into LDS once and never overwritten.
//
// Workgroup = (unit, KV head), four wavefronts that own 32 rows each.  K and V tiles of 32 tokens go from
// global memory straight into LDS (global_load_lds_dwordx4), two or three tiles before their use, with the 16-byte pieces
// of a row swizzled on the global side so that both operand reads are free of bank conflicts: K with
// ds_read_b128, V with the transposing ds_read_b64_tr_b16.  The reads are issued by hand a few fragments ahead of
// the product that takes them, with exact waits (the compiler would drain the copies before every LDS read).
//
// Tiles that every row of the workgroup sees whole run through a pipeline: one region of matrix products holds the
// scores of tile t, the probabilities of tile t - 1 and P V of tile t - 2, interleaved instruction by instruction, with
// one barrier a tile.  The others (the causal edge, a prompt's ragged end) follow one by one with the mask;
// wavefronts whose rows see nothing of such a tile skip it.
//
// Rounding: sums, statistics and accumulators are fp32, and so is what a part hands on.  The probabilities become bf16 as the second
// product's operand (2^-8 of a term; the divisor is the sum of the unrounded ones), the result bf16.
//
// Bound: the matrix pipe, and on long calls of real data its power.  64 and 8 heads of 128 channels, 16384 tokens: 3.97 to 4.11 ms, 1.07 to
// 1.12 PFLOP/s of the products that the rows need, matrix pipe 62 % busy at 1.7 GHz (2.9 ms on zeros, where the clock stays up).  128 rows a
// workgroup against 256 (half the LDS traffic, one workgroup a CU): 16384 tokens 3.98 / 3.88 ms, 2 x 8192 of 64 channels 579 / 649 us,
// 8 x 300..512 over 4k to 12k 545 / 603, 26 x 300..512 94 / 115.  Three prompts of 500 to 4001 tokens, 32 and 8 heads of 64: 107 us, 0.82
// PFLOP/s, three workgroups a CU (with 212 registers, two: 117); 2 x 4096 of 256 channels 305 us, 0.90.  4 x 17..96 new tokens over
// 2k to 8k paged ones: 40.5 us (87 MB read, 25 written), of which a unit's start is 4.3, a tile 1.0 with two units a CU, and the rows' way out 3.
#include "attn_prefix_body.h"
#include "prompt_units.h"

namespace spd {
namespace {

using prefix_impl::as_bf16x8;
using prefix_impl::bf16x8;
using prefix_impl::floatx16;
using prefix_impl::for_each_index;
using prefix_impl::pack_bf16_rne;
using prefix_impl::u32x2;
using prefix_impl::u32x4;
using prefix_impl::wait_vmcnt;
using prompt_impl::find_unit;
using prompt_impl::kRows;
using prompt_impl::Unit;

constexpr int kTileN = 32;
constexpr int kWaves = 4;
constexpr int kRing = 4;              // slots of K and of V: the tile in use and up to three under way
constexpr int kFragAhead = 4;         // LDS fragments in flight
// Tiles that some row of a workgroup does not see whole: its 128 rows end at up to 128 tokens, and a prompt's end may be ragged.
constexpr int kOddWords = 8;
constexpr float kNever = -3.402823466e38f;  // reference maximum of a row that has seen nothing: finite, so that no exponent is inf - inf
constexpr float kRaise = 1024.f;
// Reference maxima from here on (in base 2) are too large for the exponents' fma: the product there is exact and the maximum rounded, and
// the difference, up to 2^-24 of it, would go into the exponent.  Such rows take every tile's probabilities again, from rounded products.
constexpr float kLarge = 16777216.f;

template <int D> struct Shape {  // D: channels of a tile row
    static constexpr int kRow = 2 * D, kTile = kTileN * kRow;  // bytes
    static constexpr int kRowsPerCopy = 1024 / kRow, kCopies = kTile / 1024;
    static constexpr int kQK = D / 16, kDB = D / 32, kPV = 2 * kDB;  // fragments
    static constexpr int kLds = 2 * kRing * kTile + 4 * kOddWords;  // K, V, flags; 64 KB with 128 channels: two workgroups per CU
    // Piece p of a row lies in slot p ^ swz(row): sixteen rows' equal pieces take all 64 banks, and so do the four rows and
    // 64 bytes that half a wavefront's transposing reads touch.
    static __device__ __forceinline__ int swz(int row)
    {
        if (D >= 128)
            return ((row & 3) << 2) | ((row >> 2) & 3);
        return (((row >> 1) & 1) << 2) | (((row >> 2) & 1) << 1) | ((row >> 3) & 1);
    }
};

// A ring slot that is known at compile time, 0 for one that is a number.
constexpr int slot_constant(int) { return 0; }
template <int N> constexpr int slot_constant(std::integral_constant<int, N>) { return N; }

template <int D, bool FULL, bool PAGED>  // FULL: the heads have D channels, not fewer
__global__ __launch_bounds__(kWaves * 64, D <= 128 ? 2 : 1) void prompt_mfma_kernel(PromptParams p)
{
    using S = Shape<D>;
    const int head_bytes = FULL ? S::kRow : p.D * 2, head_pieces = head_bytes / 16;
    constexpr int kIPW = 2 * S::kCopies / kWaves;
    static_assert(kIPW >= 1 && kRows == 32 * kWaves, "a copy for every wavefront");
    __shared__ __align__(16) char lds[S::kLds];
    uint32_t* const odd_words = (uint32_t*)(lds + 2 * kRing * S::kTile);  // tokens whose values are not all finite, a word per such tile

    const int j = blockIdx.x % p.Hkv;
    const Unit at = find_unit(p, blockIdx.x / p.Hkv);
    if (!at.any)
        return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, h = lane >> 5;
    const int q0 = at.q0, n = at.n, L = at.L;
    const int rows = n * p.G, row0 = at.tile * kRows, rr = row0 + wave * 32 + col;
    const bool row_ok = rr < rows;
    const int token = (row_ok ? rr : 0) / p.G, head = j * p.G + (row_ok ? rr : 0) % p.G;
    const long long out_row = (long long)(q0 + token) * p.Hq + head;
    const int limit = !row_ok ? -1 : p.causal ? L - n + token : L - 1;  // the last token the row sees
    const int least = p.causal ? L - n + row0 / p.G : L - 1;
    const int most = p.causal ? L - n + (min(row0 + kRows, rows) - 1) / p.G : L - 1;
    const int wave_last = min(row0 + wave * 32 + 32, rows) - 1;  // last row of this wavefront
    const bool works = row0 + wave * 32 < rows;                     // the others copy, and wait at the barriers
    const int wave_most = !works ? -1 : p.causal ? L - n + wave_last / p.G : L - 1;

    const int seen = max(most + 1, 0);
    const int t0 = p.num_splits > 1 ? min(at.split * at.split_tokens, seen) : 0;
    const int t1 = p.num_splits > 1 ? min(t0 + at.split_tokens, seen) : seen;
    const int ntiles = (t1 - t0 + kTileN - 1) / kTileN;
    const int whole = max(min(least + 1, t1) - t0, 0) / kTileN;  // tiles that every row sees whole
    const int nfull = whole < 3 ? 0 : whole;                      // those that run through the pipeline

    // ---- query fragments (B operand): column = this lane's row, channels 16 s + 8 h (a lane without a row of its own takes
    // the first token's: nothing of it is stored)
    bf16x8 qf[S::kQK];
    {
        const uint4* qg = (const uint4*)((const char*)p.q + ((long long)(q0 + token) * p.q_stride + (long long)head * (head_bytes / 2)) * 2);
#pragma unroll
        for (int s = 0; s < S::kQK; ++s) {
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (FULL || 2 * s + h < head_pieces)
                v = qg[2 * s + h];
            qf[s] = as_bf16x8(v);
        }
    }

    // ---- global -> LDS copies: the first half of the wavefronts copies K, the other half V, kIPW instructions a tile each
    typedef const __attribute__((address_space(4))) int* const_int_ptr;
    const const_int_ptr pages = PAGED ? (const_int_ptr)(p.pages + at.kv0) : nullptr;
    const long long tok_stride = PAGED ? head_bytes : p.kv_stride * 2;
    const long long head_base = PAGED ? (long long)j * 16 * head_bytes : (long long)at.kv0 * p.kv_stride * 2 + (long long)j * head_bytes;
    const long long page_stride = (long long)p.Hkv * 16 * head_bytes;
    const unsigned lds_base = (unsigned)(size_t)(__attribute__((address_space(3))) void*)lds;
    constexpr int kLanesPerRow = 64 / S::kRowsPerCopy;
    const int lane_row = lane / kLanesPerRow, lane_piece = lane % kLanesPerRow;
    const bool copies_v = wave >= kWaves / 2;
    const int row_first = S::kRowsPerCopy * kIPW * (copies_v ? wave - kWaves / 2 : wave);
    // piece of its row that this lane fetches with instruction i
    auto piece_of = [&](int i) __attribute__((always_inline)) { return lane_piece ^ S::swz(row_first + S::kRowsPerCopy * i + lane_row); };
    unsigned lane_off[kIPW];
#pragma unroll
    for (int i = 0; i < kIPW; ++i)
        lane_off[i] = (unsigned)((S::kRowsPerCopy * i + lane_row) * (unsigned)tok_stride + (piece_of(i) << 4));
    const char* const tensor = (const char*)(copies_v ? p.v : p.k);
    char* const ring_lds = lds + (copies_v ? kRing * S::kTile : 0) + row_first * S::kRow;
    int next_page = 0;
    auto fetch_page = [&](int tile) __attribute__((always_inline)) {
        if (PAGED)
            next_page = pages[min(t0 + tile * kTileN + row_first, t1 - 1) >> 4];
    };
    int issued = -1;  // last tile whose copies this wavefront has started
    auto issue_next = [&]() __attribute__((always_inline)) {
        const int tile = ++issued, tb = t0 + tile * kTileN;
        char* const dst = ring_lds + (tile % kRing) * S::kTile;
        const bool full = tb + kTileN <= t1;
        const int tg = min(tb + row_first, t1 - 1);  // this wavefront's first row; rows past the end repeat the last token
        const char* const src = PAGED ? tensor + (long long)next_page * page_stride + head_base + (tg & 15) * head_bytes
                                      : tensor + head_base + (long long)tg * tok_stride;
#pragma unroll
        for (int i = 0; i < kIPW; ++i) {
            unsigned off = lane_off[i];
            if (!full) {
                const int tl = S::kRowsPerCopy * i + lane_row, row = min(tb + row_first + tl, t1 - 1) - tg;
                off = (unsigned)(max(row, 0) * (unsigned)tok_stride + (piece_of(i) << 4));
            }
            if (FULL || piece_of(i) < head_pieces)  // (every instruction has lanes that copy)
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src + off),
                                             (__attribute__((address_space(3))) void*)(dst + i * 1024), 16, 0, 0);
        }
        fetch_page(tile + 1);
    };
    auto copies_up_to = [&](int tile) __attribute__((always_inline)) {
#pragma unroll 1
        while (issued < min(tile, ntiles - 1))
            issue_next();
    };
    // Waits until this wavefront's copies of `tile` have landed (later ones may be under way), then for everybody.
    auto landed = [&](int tile) __attribute__((always_inline)) {
        const int later = issued - tile;
        if (later >= 2)
            wait_vmcnt<2 * kIPW>();
        else if (later == 1)
            wait_vmcnt<kIPW>();
        else
            wait_vmcnt<0>();
        __builtin_amdgcn_s_barrier();
    };

    // ---- per-lane LDS addresses of the operand fragments in slot 0; the slot goes into the instruction's offset, and so do
    // the second 256 bytes of a row, whose swizzle is the first's
    constexpr int kAddrK = S::kQK < 8 ? S::kQK : 8, kAddrV = S::kDB < 4 ? S::kDB : 4;
    unsigned k_addr[kAddrK], v_addr[kAddrV][2];
#pragma unroll
    for (int s = 0; s < kAddrK; ++s)
        k_addr[s] = lds_base + (unsigned)(col * S::kRow) + ((32u * s) ^ (unsigned)((h ^ S::swz(col)) << 4));
    {
        const int g16 = (lane >> 4) & 1, r = (lane & 15) >> 2, q4 = lane & 3;
#pragma unroll
        for (int db = 0; db < kAddrV; ++db)
#pragma unroll
            for (int part2 = 0; part2 < 2; ++part2) {
                const int tok = 8 * part2 + 4 * h + r, piece = 4 * db + 2 * g16 + (q4 >> 1);
                v_addr[db][part2] = lds_base + (unsigned)(kRing * S::kTile + tok * S::kRow + ((piece ^ S::swz(tok)) << 4) + (q4 & 1) * 8);
            }
    }

    float m_run = kNever, l_run = 0.f, sum_cap = kRaise;
    floatx16 o[S::kDB];
#pragma unroll
    for (int db = 0; db < S::kDB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i)
            o[db][i] = 0.f;

    u32x4 ring_k[kFragAhead + 2];
    u32x2 ring_lo[kFragAhead + 2], ring_hi[kFragAhead + 2];
    // One region: scores of the tile in K slot `kslot` into `sn` (QK), P V of the tile in V slot `vslot` with
    // probabilities `pp` (PV; the two products alternate; slots are constants or numbers), and between the products the probabilities `pn` of the scores `so` (SM; their sum over the
    // lane is returned).
    auto region = [&](auto qk_tag, auto sm_tag, auto pv_tag, auto kslot, auto vslot, floatx16& sn, const floatx16& so,
                      bf16x8 (&pn)[2], const bf16x8 (&pp)[2]) __attribute__((always_inline)) -> float {
        constexpr bool QK = decltype(qk_tag)::value, SM = decltype(sm_tag)::value, PV = decltype(pv_tag)::value;
        constexpr bool kBoth = QK && PV;
        static_assert(S::kQK == S::kPV, "as many fragments of either product");
        constexpr int NF = (QK ? S::kQK : 0) + (PV ? S::kPV : 0);
        if (QK) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                sn[i] = 0.f;
        }
        auto issue = [&](auto kc) __attribute__((always_inline)) {
            constexpr int K = decltype(kc)::value;
            if constexpr (K < NF) {
                constexpr int idx = kBoth ? K >> 1 : K;
                constexpr bool is_pv = kBoth ? (K & 1) != 0 : PV;
                constexpr bool fixed = !std::is_same<decltype(kslot), int>::value;
                if constexpr (!is_pv) {
                    u32x4& dst = ring_k[K % (kFragAhead + 2)];
                    unsigned addr = k_addr[idx % kAddrK];
                    constexpr int kSlot = slot_constant(decltype(kslot){}) * S::kTile;
                    if constexpr (!fixed)
                        addr += (unsigned)kslot * S::kTile;
                    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(dst) : "v"(addr), "n"(kSlot + idx / kAddrK * 256));
                } else {
                    constexpr int a = idx / S::kDB, b = idx % S::kDB;
                    u32x2& lo = ring_lo[K % (kFragAhead + 2)];
                    u32x2& hi = ring_hi[K % (kFragAhead + 2)];
                    unsigned a0 = v_addr[b % kAddrV][0], a1 = v_addr[b % kAddrV][1];
                    constexpr int kSlot = slot_constant(decltype(vslot){}) * S::kTile;
                    if constexpr (!fixed) {
                        a0 += (unsigned)vslot * S::kTile;
                        a1 += (unsigned)vslot * S::kTile;
                    }
                    asm volatile("ds_read_b64_tr_b16 %0, %2 offset:%4\n\tds_read_b64_tr_b16 %1, %3 offset:%4"
                                 : "=&v"(lo), "=&v"(hi)
                                 : "v"(a0), "v"(a1), "n"(kSlot + a * 16 * S::kRow + b / kAddrV * 256));
                }
            }
        };
        auto consume = [&](auto kc) __attribute__((always_inline)) {
            constexpr int K = decltype(kc)::value;
            constexpr int idx = kBoth ? K >> 1 : K;
            constexpr bool is_pv = kBoth ? (K & 1) != 0 : PV;
            // LDS instructions issued after fragment K
            constexpr int last = K + kFragAhead < NF ? K + kFragAhead : NF - 1;
            constexpr int later = last - K;
            constexpr int after = kBoth ? later + (is_pv ? later / 2 : (later + 1) / 2) : PV ? 2 * later : later;
            if constexpr (!is_pv) {
                u32x4& f = ring_k[K % (kFragAhead + 2)];
                asm volatile("s_waitcnt lgkmcnt(%1)" : "+v"(f) : "n"(after));
                sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(f), qf[idx], sn, 0, 0, 0);
            } else {
                u32x2& lo = ring_lo[K % (kFragAhead + 2)];
                u32x2& hi = ring_hi[K % (kFragAhead + 2)];
                asm volatile("s_waitcnt lgkmcnt(%2)" : "+v"(lo), "+v"(hi) : "n"(after));
                const u32x4 f = {lo[0], lo[1], hi[0], hi[1]};
                constexpr int a = idx / S::kDB, b = idx % S::kDB;
                o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(f), pp[a], o[b], 0, 0, 0);
            }
        };
        // Slot e of the softmax: the exponent of score e, the exponential of score e - 1, the sum of score e - 2.
        float psum = 0.f, x[16], pv[16];
        uint32_t w[8];
        auto soft = [&](auto ec) __attribute__((always_inline)) {
            constexpr int e = decltype(ec)::value;
            if constexpr (SM && e >= 0 && e < 18) {
                if constexpr (e < 16)
                    x[e] = __builtin_fmaf(so[e], p.scale_log2, -m_run);
                if constexpr (e >= 1 && e < 17)
                    pv[e - 1] = __builtin_amdgcn_exp2f(x[e - 1]);
                if constexpr (e >= 2) {
                    psum += pv[e - 2];
                    if constexpr ((e & 1) != 0)
                        w[(e - 2) >> 1] = pack_bf16_rne(pv[e - 3], pv[e - 2]);
                }
            }
        };
        constexpr int kPer = 18 / NF > 0 ? 18 / NF : 1, kLead = kPer * NF < 18 ? 18 - kPer * NF : 0;  // slots per product, and before the first
        for_each_index(issue, std::make_integer_sequence<int, kFragAhead + 1>{});
        if constexpr (SM) {
            for_each_index(soft, std::make_integer_sequence<int, kLead>{});
            __builtin_amdgcn_sched_barrier(0);
        }
        for_each_index(
            [&](auto kc) __attribute__((always_inline)) {
                constexpr int K = decltype(kc)::value;
                consume(kc);
                issue(std::integral_constant<int, K + kFragAhead + 1>{});
                if constexpr (SM) {
                    for_each_index([&](auto ic) __attribute__((always_inline)) {
                        soft(std::integral_constant<int, K * kPer + decltype(ic)::value + kLead>{});
                    }, std::make_integer_sequence<int, kPer>{});
                    __builtin_amdgcn_sched_barrier(0);
                }
            },
            std::make_integer_sequence<int, NF>{});
        if constexpr (SM) {
            const uint4 p0 = make_uint4(w[0], w[1], w[2], w[3]), p1 = make_uint4(w[4], w[5], w[6], w[7]);
            pn[0] = as_bf16x8(p0);
            pn[1] = as_bf16x8(p1);
        }
        return psum;
    };

    auto probabilities = [&](auto rounded, const floatx16& sc, bf16x8 (&pn)[2]) __attribute__((always_inline)) -> float {
#pragma clang fp contract(off)
        float psum = 0.f;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            float pv[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = sc[8 * u + e];
                pv[e] = __builtin_amdgcn_exp2f(decltype(rounded)::value ? x * p.scale_log2 - m_run : __builtin_fmaf(x, p.scale_log2, -m_run));
                psum += pv[e];
            }
            uint4 pu;
            pu.x = pack_bf16_rne(pv[0], pv[1]);
            pu.y = pack_bf16_rne(pv[2], pv[3]);
            pu.z = pack_bf16_rne(pv[4], pv[5]);
            pu.w = pack_bf16_rne(pv[6], pv[7]);
            pn[u] = as_bf16x8(pu);
        }
        return psum;
    };
    // The reference maximum only has to bound the exponents: it is raised where a lane's 16 probabilities add up to more
    // than kRaise (none is above that otherwise: exact in fp32 and bf16 alike), or where it is kLarge.  O holds every earlier tile by then.
    auto raise_maximum = [&](const floatx16& sc) __attribute__((always_inline)) -> float {
        float tmax = kNever;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            tmax = fmaxf(tmax, sc[i] * p.scale_log2);
        tmax = fmaxf(tmax, __shfl_xor(tmax, 32));
        const float m_up = fmaxf(m_run, tmax);
        const float corr = __builtin_amdgcn_exp2f(m_run - m_up);
        m_run = m_up;
        sum_cap = fabsf(m_up) >= kLarge && m_up != kNever ? -1.f : kRaise;
        return corr;
    };
    auto take_sum = [&](float psum, const floatx16& sc, bf16x8 (&pn)[2]) __attribute__((always_inline)) {
        if (__ballot(!(psum <= sum_cap)) != 0) {
            const float corr = raise_maximum(sc);
            psum = probabilities(std::true_type{}, sc, pn);
            l_run *= corr;
#pragma unroll
            for (int db = 0; db < S::kDB; ++db) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    o[db][i] *= corr;
                if (D > 128)
                    __builtin_amdgcn_sched_barrier(0);  // (one block at a time out of the accumulation registers)
            }
        }
        l_run += psum;
    };

    // ---- the pipeline ---------------------------------------------------------------------------------------------------
    // Step t starts the copies of K of tile t + 3 and V of tile t + 1 (into slots that a barrier has freed: K of tile t - 1, V of
    // tile t - 3), runs its region (scores of tile t, P V of tile t - 2), and waits until K of tile t + 1 and V of tile t - 1 have
    // landed for everybody.  The four slots make four steps one round of the loop.
    const std::true_type yes{};
    const std::false_type no{};
    floatx16 sa, sb;
    bf16x8 pa[2], pb[2];
    const int lead = copies_v && nfull > 0 ? 1 : 3, lag = copies_v ? 1 : -1;
    if (ntiles > 0) {
        if (tid < kOddWords)
            odd_words[tid] = 0u;  // (a barrier follows before any is set)
        if (!FULL) {
            for (int i = tid; i < 2 * kRing * S::kTile / 16; i += kWaves * 64)
                reinterpret_cast<uint4*>(lds)[i] = make_uint4(0u, 0u, 0u, 0u);
            __syncthreads();
        }
        fetch_page(0);
        copies_up_to(lead - 1);
        landed(0);
    }
    int t = 0;
    if (nfull > 0) {
        // One step with its slots as constants: the scores of even tiles are in sa, those of odd ones in sb.
        auto step = [&](auto tc) __attribute__((always_inline)) {
            constexpr int T = decltype(tc)::value;
            const std::integral_constant<int, T % kRing> kslot;
            const std::integral_constant<int, (T + 2) % kRing> vslot;
            copies_up_to(t + lead);
            if (!works) {
            } else if constexpr (T % 2 == 0)
                take_sum(region(yes, yes, yes, kslot, vslot, sa, sb, pb, pa), sb, pb);
            else
                take_sum(region(yes, yes, yes, kslot, vslot, sb, sa, pa, pb), sa, pa);
            landed(t - lag);
            ++t;
        };
        copies_up_to(lead);
        region(yes, no, no, std::integral_constant<int, 0>{}, std::integral_constant<int, 0>{}, sa, sa, pa, pa);
        landed(copies_v ? 0 : 1);
        raise_maximum(sa);
        copies_up_to(1 + lead);
        take_sum(region(yes, yes, no, std::integral_constant<int, 1>{}, std::integral_constant<int, 0>{}, sb, sa, pa, pb), sa, pa);
        landed(1 - lag);
        t = 2;
        while (true) {  // (nfull > 2)
            step(std::integral_constant<int, 2>{});
            if (t >= nfull)
                break;
            step(std::integral_constant<int, 3>{});
            if (t >= nfull)
                break;
            step(std::integral_constant<int, 0>{});
            if (t >= nfull)
                break;
            step(std::integral_constant<int, 1>{});
            if (t >= nfull)
                break;
        }
        // The scores of tile t - 1 and the probabilities of tile t - 2 are left; V of tile t - 2 has landed.
        if (t & 1) {
            sb = sa;
            pa[0] = pb[0];
            pa[1] = pb[1];
        }
        copies_up_to(t + (copies_v ? 1 : 2));
        take_sum(region(no, yes, yes, 0, (t - 2) % kRing, sa, sb, pb, pa), sb, pb);
        landed(copies_v ? t - 1 : min(t, ntiles - 1));
        copies_up_to(t + 2);
        region(no, no, yes, 0, (t - 1) % kRing, sa, sa, pa, pb);
        landed(min(t, ntiles - 1));
    }

    // ---- tiles that some row does not see whole ------------------------------------------------------------------------------
    for (; t < ntiles; ++t) {
        const int tb = t0 + t * kTileN, slot = t % kRing;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        copies_up_to(t + 3);  // (the slots of tile t - 1 are free for everybody from here on)
        const bool some = tb <= wave_most;
        const bool masked = t >= whole;
        if (masked) {
            // 0 * inf is not 0: values that are not finite are noted, taken out of the tile, and added at the end to the rows that
            // see them.  (The tile's copies have landed.)
            for (int i = tid; i < S::kTile / 16; i += kWaves * 64) {
                uint4* const at_piece = reinterpret_cast<uint4*>(lds + (kRing + slot) * S::kTile) + i;
                uint4 v;
                const unsigned addr = lds_base + (unsigned)(kRing + slot) * S::kTile + i * 16;
                u32x4 raw;
                asm volatile("ds_read_b128 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=v"(raw) : "v"(addr));
                uint32_t w[4];
                bool any = false;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool lo = (raw[e] & 0x7f80u) == 0x7f80u, hi = (raw[e] & 0x7f800000u) == 0x7f800000u;
                    w[e] = raw[e] & (lo ? 0xffff0000u : 0xffffffffu) & (hi ? 0x0000ffffu : 0xffffffffu);
                    any = any || lo || hi;
                }
                if (any) {
                    atomicOr(&odd_words[min(t - whole, kOddWords - 1)], 1u << (i / (S::kRow / 16)));
                    v = make_uint4(w[0], w[1], w[2], w[3]);
                    *at_piece = v;
                }
            }
        }
        if (some) {
            region(yes, no, no, slot, 0, sa, sa, pa, pa);
            if (masked) {
                const int end = min(limit, t1 - 1) - tb - 4 * h;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    sa[i] = 8 * (i >> 2) + (i & 3) <= end ? sa[i] : -INFINITY;
            }
            take_sum(probabilities(no, sa, pa), sa, pa);
        }
        if (masked) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
        }
        if (some)
            region(no, no, yes, 0, slot, sa, sa, pa, pa);
        if (t + 1 < ntiles)
            landed(t + 1);
    }

    // ---- results: through LDS (the rings are free), so that a row leaves in whole lines ------------------------------------
    const float l = l_run + __shfl_xor(l_run, 32);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    __builtin_amdgcn_s_barrier();
    // Rows 0 .. 31 of the wavefront to `first` + out_row * `pitch`: a result's, in bf16, or a part's sums as they are, whose rows are twice as
    // long and take the rings to their last byte.
    auto store_rows = [&](auto sums_tag, char* first, long long pitch) __attribute__((always_inline)) {
        constexpr bool SUMS = decltype(sums_tag)::value;
        constexpr int kBytes = SUMS ? 2 * S::kRow : S::kRow, kPieces = kBytes / 16, kRowsAtOnce = 64 / kPieces;
        char* const mine = lds + wave * 32 * kBytes;
        auto place = [&](int row, int piece) __attribute__((always_inline)) -> char* {
            return mine + row * kBytes + ((piece ^ (row & (kPieces - 1))) << 4);
        };
#pragma unroll
        for (int db = 0; db < S::kDB; ++db)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {  // registers 4 q4 .. + 3 are channels 32 db + 8 q4 + 4 h .. + 3
                const float x0 = o[db][4 * q4], x1 = o[db][4 * q4 + 1], x2 = o[db][4 * q4 + 2], x3 = o[db][4 * q4 + 3];
                if constexpr (SUMS)
                    *reinterpret_cast<float4*>(place(col, 8 * db + 2 * q4 + h)) = make_float4(x0, x1, x2, x3);
                else
                    *reinterpret_cast<uint2*>(place(col, 4 * db + q4) + 8 * h) =
                        make_uint2(pack_bf16_rne(x0 * inv, x1 * inv), pack_bf16_rne(x2 * inv, x3 * inv));
            }
        // rare: the values that were taken out of the tiles, to the rows that see them
        for (int w = 0; w < kOddWords; ++w)
            for (uint32_t bits = ntiles > 0 ? __builtin_amdgcn_readfirstlane(odd_words[w]) : 0u; bits != 0u; bits &= bits - 1u) {
                const int x = t0 + (whole + w) * kTileN + __ffs(bits) - 1;
                if (x >= t1)
                    continue;
                const uint16_t* v = (const uint16_t*)((const char*)p.v + head_base + (PAGED ? (long long)pages[x >> 4] * page_stride + (x & 15) * head_bytes
                                                                                              : (long long)x * tok_stride));
                for (int row = 0; row < 32; ++row) {
                    if (x > __builtin_amdgcn_readfirstlane(__shfl(limit, row)))
                        continue;
                    for (int c = lane; c < head_bytes / 2; c += 64) {
                        const float value = __uint_as_float((uint32_t)v[c] << 16);
                        if (fabsf(value) < INFINITY)
                            continue;
                        if constexpr (SUMS) {
                            reinterpret_cast<float*>(place(row, c >> 2))[c & 3] += value;
                        } else {
                            uint16_t* const at_c = reinterpret_cast<uint16_t*>(place(row, c >> 3)) + (c & 7);
                            *at_c = (uint16_t)pack_bf16_rne(__uint_as_float((uint32_t)*at_c << 16) + value, 0.f);
                        }
                    }
                }
            }
        const int to = row_ok ? (int)out_row : -1, at_row = lane / kPieces, piece = lane % kPieces;
#pragma unroll
        for (int i = 0; i < 32 / kRowsAtOnce; ++i) {
            const int row = kRowsAtOnce * i + at_row, dst = __shfl(to, row);
            if (dst >= 0 && (FULL || piece < head_pieces * (SUMS ? 2 : 1)))
                *reinterpret_cast<uint4*>(first + dst * pitch + piece * 16) = *reinterpret_cast<const uint4*>(place(row, piece));
        }
    };
    if (p.num_splits > 1) {
        if (h == 0 && row_ok) {
            p.part_ml[out_row * p.num_splits + at.split] = make_float4(m_run, l, 0.f, 0.f);
            if (at.split == 0)  // and the parts that this prompt does not have
                for (int s = at.splits; s < p.num_splits; ++s)
                    p.part_ml[out_row * p.num_splits + s] = make_float4(kNever, 0.f, 0.f, 0.f);
        }
        if (t0 < t1)
            store_rows(yes, (char*)p.part_acc + (long long)at.split * p.D * 4, (long long)p.num_splits * p.D * 4);
        return;
    }
    if (p.lse && h == 0 && row_ok)
        p.lse[out_row] = l == 0.f ? -INFINITY : m_run * kLn2 + logf(l);
    store_rows(no, (char*)p.out, head_bytes);
}

template <int D, bool FULL> void launch(const PromptParams& p, hipStream_t s)
{
    const dim3 grid((unsigned)((long long)p.tiles * p.num_splits * p.Hkv)), block(kWaves * 64);
    if (p.page_size != 0)
        hipLaunchKernelGGL((prompt_mfma_kernel<D, FULL, true>), grid, block, 0, s, p);
    else
        hipLaunchKernelGGL((prompt_mfma_kernel<D, FULL, false>), grid, block, 0, s, p);
}

template <int D> void launch(const PromptParams& p, hipStream_t s)
{
    p.D == D ? launch<D, true>(p, s) : launch<D, false>(p, s);
}

}  // namespace

hipError_t launch_prompt_mfma(const PromptParams& p, hipStream_t s)
{
    p.D <= 64 ? launch<64>(p, s) : p.D <= 128 ? launch<128>(p, s) : launch<256>(p, s);
    return hipGetLastError();
}

}  // namespace spd
