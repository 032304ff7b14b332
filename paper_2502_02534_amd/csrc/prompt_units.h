// Which piece of a prompt_attn call a workgroup takes, shared by its kernels.
//
// Work is cut into units: (prompt, tile of kPromptRows rows, part of split_tokens tokens), times the KV heads.  The
// host knows only bounds on the lengths, so the units of each prompt are counted on the device, by every wavefront
// for itself: 64 prompts at a time, a lane each, with everything about the prompt that the workgroup needs.  They follow
// one another prompt by prompt, or (a few causal prompts) by the number of their tile, last tiles first.
//
// Parts.  A part costs its rows' partial states (written once, read once by the launch that joins them) besides a workgroup's
// start, so there are no more than run at once: with W = sum of tiles * tokens and T = number of tiles, over all KV heads,
// parts of W / (kPlaces - T) tokens are at most kPlaces, because a prompt's last part is the only one that is not full.
#pragma once

#include "spd_internal.h"

namespace spd {
namespace prompt_impl {

constexpr int kRows = 128;   // (new token, head of the group) rows per workgroup
constexpr int kPlaces = 512; // workgroups that run at once: two a CU

struct Unit {
    bool any;           // false: past the last unit
    int q0, n, L, kv0;  // the prompt's first query and their number, its tokens, its place in the KV table
    int tile;           // the prompt's last tiles, which see most, come first; where all units run at once, two a CU (unit i and unit
                        // i + half of them), those of the second half come last, so that pairs are even
    int split, splits;  // of the prompt's tokens
    int split_tokens;
};

__device__ __forceinline__ int row_tiles(const PromptParams& p, int n) { return (n * p.G + kRows - 1) / kRows; }

__device__ __forceinline__ Unit find_unit(const PromptParams& p, int item)
{
    const int lane = threadIdx.x & 63;
    Unit u;
    u.any = false;
    u.q0 = u.n = u.L = u.kv0 = u.tile = u.split = 0;
    u.splits = 1;
    u.split_tokens = 0;
    int q0, n, L, kv0, tiles;  // of the lane's prompt
    auto load = [&](int b0) __attribute__((always_inline)) {
        const int b = min(b0 + lane, p.B - 1);
        q0 = p.query_indptr[b];
        const int q1 = p.query_indptr[b + 1];
        L = p.kv_lens[b];
        kv0 = p.kv_indptr[b];
        n = max(q1 - q0, 0);
        tiles = b0 + lane < p.B ? row_tiles(p, n) : 0;
    };
    load(0);
    const auto of = [](int x, int l) { return __builtin_amdgcn_readlane(x, l); };
    const auto take = [&](int l) __attribute__((always_inline)) {
        u.any = true;
        u.q0 = of(q0, l);
        u.n = of(n, l);
        u.L = of(L, l);
        u.kv0 = of(kv0, l);
    };
    if (p.by_length) {
        // with `ahead(t)` the units of tiles t and later, the largest t with ahead(t) > item, 64 candidates at a time
        int lo = 0, width = p.tiles + 1, ahead = 0;
        while (width > 1) {
            const int step = (width + 63) >> 6, t = lo + lane * step;
            int here = 0;
            for (int b = 0; b < p.B; ++b)
                here += max(of(tiles, b) - t, 0);
            const unsigned long long fits = __ballot(here > item);
            if (fits == 0ull)
                return u;  // past the last unit (the first candidate counts them all)
            const int l = 63 - __clzll((long long)fits);
            ahead = of(here, l);
            lo += l * step;
            width = step;
        }
        const unsigned long long have = __ballot(tiles > lo);
        const int nth = item - (ahead - __popcll(have));  // among the prompts that have this tile
        const int rank = __builtin_amdgcn_mbcnt_hi((unsigned)(have >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)have, 0u));
        take(__ffsll(__ballot(tiles > lo && rank == nth)) - 1);
        u.tile = lo;
        return u;
    }
    if (p.num_splits > 1) {
        // tokens of a part: the same in every lane of every wavefront
        float work = (float)tiles * (float)max(L, 0), all = (float)tiles;
        for (int b0 = 64; b0 < p.B; b0 += 64) {
            load(b0);
            work += (float)tiles * (float)max(L, 0);
            all += (float)tiles;
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            work += __shfl_xor(work, o);
            all += __shfl_xor(all, o);
        }
        const float parts = fmaxf((float)kPlaces - all * (float)p.Hkv, 1.f);
        const int tokens = ((int)fminf(work * (float)p.Hkv / parts, 1e9f) + 32) & ~31;
        u.split_tokens = __builtin_amdgcn_readfirstlane(max(tokens, p.split_tokens));
    }
    int base = 0;
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        if (p.B > 64)
            load(b0);
        const int splits = p.num_splits > 1 ? min(max((L + u.split_tokens - 1) / u.split_tokens, 1), p.num_splits) : 1;
        const int units = tiles * splits;
        int upto = units;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int x = __shfl_up(upto, o);
            upto += lane >= o ? x : 0;
        }
        const int all = __builtin_amdgcn_readfirstlane(__shfl(upto, 63));
        if (item < base + all) {
            const int l = __ffsll((unsigned long long)__ballot(item < base + upto)) - 1;
            take(l);
            u.splits = of(splits, l);
            // the tiles of a part follow one another: they read the same tokens
            const int start = base + of(upto - units, l), local = item - start, t = of(tiles, l);
            const int i = local % t;
            u.split = local / t;
            u.tile = t - 1 - i;
            if (p.paired) {
                const int half = p.tiles / 2;
                if (start >= half)
                    u.tile = i;
                else if (start + t > half && i >= half - start)
                    u.tile = i - (half - start);
            }
            break;
        }
        base += all;
    }
    return u;
}

}  // namespace prompt_impl
}  // namespace spd
