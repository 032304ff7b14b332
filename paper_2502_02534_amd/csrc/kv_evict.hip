// Which tokens of a cache stay (select_kv_tokens), and the copies that bring them together (compact_kv).
//
// Selection.  A row's weights lie in registers, as whole numbers in their order; token = 64 (V wave + v) + lane, so that a ballot
// has 64 tokens in their order.  The c-th largest of those that are not kept by their place: a histogram in LDS of the first 9 or 11
// bits above the lowest, then the others, bit by bit, of the few keys that share them, until exactly c reach the number (then nobody
// asks which ties stay).  From there on a group of 64 tokens is 64 bits of one lane: gaps among the early places and tokens that move are counted
// for all groups at once, the tokens that move are listed in LDS in their order, and the gaps take them from there, in loops over the groups that
// have any (in straight lines from the ballots, group by group: 15.6 us instead of 10.6 for 8 rows of 16384).  Rows of up to 2048 tokens take a wavefront, longer ones a workgroup; beyond what its
// registers hold (32768), the c-th largest comes from four histograms over memory.
// Bound: issue, of the vector and the scalar unit alike, and one round of wavefronts: 8192 rows of up to 2048 weights 22 to 23 us (59 MB; bit by bit
// from the first on 37), 8 rows of 16384 10.6, 16 of 32768 15.7.
//
// Compaction.  source[i] >= i, so a workgroup that takes its places in ascending order, and reads every group of
// places before it writes them, overwrites nothing that it still has to read; where no source of a row lies below its new length the
// order does not matter, nobody waits, and few long rows are cut into stretches of places.  Only tokens that move are touched.  Bound: HBM, what moves read and written once: 1024 samples
// of up to 2048 tokens, 8 heads of 128 bf16 channels, down to 1024: 312 us (1.44 GB, 4.6 TB/s); 8 prompts of 1k to 16k down to a quarter, into
// other pages, 42 (148 MB), in place 32 (one workgroup for every piece of a row instead of stretches 65); 29 fp32 rows of up to 10k down to three
// quarters 19 (54).
#include "spd_internal.h"

namespace spd {
namespace {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;  // of the kernels without a choice
constexpr int kLong = 1024;    // of rows that no registers hold

// Weights as whole numbers in their order; NaN below all.
__device__ __forceinline__ unsigned key_of(float w)
{
    const int u = __float_as_int(w + 0.f);  // (both zeros are one value)
    return w != w ? 1u : (unsigned)(u ^ (u >> 31 | (int)0x80000000));  // (0: no token)
}

__device__ __forceinline__ int lanes_below(unsigned long long mask)
{
    return __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0u));
}

// The lowest n of 64 bits.
__device__ __forceinline__ unsigned long long lowest_bits(int n)
{
    return n >= 64 ? ~0ull : (1ull << max(n, 0)) - 1ull;
}

// Over the 16 lanes of a lane row (rotations by 8, 4, 2, 1; shifts by 1, 2, 4, 8 with zeros behind).
template <int CTRL> __device__ __forceinline__ unsigned dpp(unsigned x)
{
    return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true);
}
template <class F> __device__ __forceinline__ unsigned over_row(unsigned x, F f)
{
    x = f(x, dpp<0x128>(x));
    x = f(x, dpp<0x124>(x));
    x = f(x, dpp<0x122>(x));
    return f(x, dpp<0x121>(x));
}
template <class F> __device__ __forceinline__ unsigned over_wave(unsigned x, F f)
{
    x = over_row(x, f);
    const auto of = [&](int lane) { return (unsigned)__builtin_amdgcn_readlane((int)x, lane); };
    return f(f(of(0), of(16)), f(of(32), of(48)));
}
// Sum of the lanes up to this one, of lanes 0 .. 31.
__device__ __forceinline__ unsigned up_to_lane(unsigned x)
{
    x += dpp<0x111>(x);
    x += dpp<0x112>(x);
    x += dpp<0x114>(x);
    x += dpp<0x118>(x);
    const unsigned first = (unsigned)__builtin_amdgcn_readlane((int)x, 15);
    return x + ((threadIdx.x & 16) ? first : 0u);
}
__device__ __forceinline__ unsigned long long lane_bits(unsigned long long x, int lane)
{
    return (unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((int)x, lane);
}

// What stays of a row: n tokens, m places, the last r and the first f by their place, c of those between by weight.
struct Row {
    int n, m, r, f, c;
};

__device__ __forceinline__ Row row_of(const SelectParams& p, long long b)
{
    Row w;
    w.n = max(min(p.lens[b], p.max_len), 0);
    w.m = min(w.n, p.budgets ? max(min(p.budgets[b], p.max_new), 0) : p.max_new);
    w.r = min(p.recent, w.m);
    w.f = min(p.sinks, w.m - w.r);
    w.c = w.m - w.r - w.f;
    return w;
}

// WAVES wavefronts a row, V weights a lane; ROWS rows a workgroup (1 where WAVES > 1).
template <int WAVES, int V, int ROWS> __global__ __launch_bounds__(64 * WAVES * ROWS) void select_rows(SelectParams p)
{
    constexpr int kTokens = 64 * WAVES * V;
    constexpr int kBits = V < 16 ? 0 : WAVES == 1 ? 9 : 11;  // of the histogram
    constexpr int kBins = 1 << kBits, kOwn = kBins < 64 ? 1 : kBins / 64;  // and a lane's bins of it, with a place between two lanes' (bank conflicts)
    constexpr int kPlaces = kBins + 128;
    const auto place = [](int bin) { return bin + bin / kOwn; };
    static_assert(WAVES == 1 || ROWS == 1, "wavefronts of one row wait for each other");
    __shared__ unsigned short moving[ROWS][kTokens / 2];  // (no more than half of the tokens fill gaps)
    __shared__ int counts[2][WAVES], sums[2][WAVES];
    __shared__ __align__(16) int hist[kBits ? ROWS : 1][kBits ? kPlaces : 4];
    __shared__ unsigned few[ROWS][64];
    __shared__ int num_few;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int w = WAVES == 1 ? 0 : wave, local = WAVES == 1 ? wave : 0;
    const long long row = (long long)blockIdx.x * ROWS + local;
    if (row >= p.seqs * p.heads)
        return;
    const Row a = row_of(p, row / p.heads);
    int* const source = p.source + row * p.source_stride;
    if (row % p.heads == 0 && threadIdx.x % (64 * WAVES) == 0)
        p.new_lens[row / p.heads] = a.m;
    const int t0 = 64 * V * w;  // this wavefront's first token
    if (a.m == a.n) {
#pragma unroll 4
        for (int v = 0; v < V; ++v)
            if (t0 + 64 * v + lane < a.m)
                source[t0 + 64 * v + lane] = t0 + 64 * v + lane;
        return;
    }
    const float* const weights = p.weights + row * p.stride;
    const int middle = a.n - a.r, early = a.m - a.r;  // tokens f .. middle - 1 are chosen from; places before `early` have gaps
    // (four groups of 64 tokens at a time, as far as there are any)
    float x[V];
#pragma unroll
    for (int v0 = 0; v0 < V; v0 += 4)
        if (t0 + 64 * v0 < middle) {
#pragma unroll
            for (int v = v0; v < v0 + 4; ++v) {
                const int t = t0 + 64 * v + lane;
                x[v] = weights[min(max(t, a.f), middle - 1)];
            }
        }
    unsigned key[V];
    unsigned lowest = ~0u, highest = 0u;  // (less one)
#pragma unroll
    for (int v0 = 0; v0 < V; v0 += 4) {
        if (t0 + 64 * v0 < middle) {
#pragma unroll
            for (int v = v0; v < v0 + 4; ++v) {
                key[v] = (unsigned)(t0 + 64 * v + lane - a.f) < (unsigned)(middle - a.f) ? key_of(x[v]) : 0u;
                lowest = min(lowest, key[v] - 1u);
                highest = max(highest, key[v]);
            }
        } else {
#pragma unroll
            for (int v = v0; v < v0 + 4; ++v)
                key[v] = 0u;
        }
    }
    // a number over the row's wavefronts (every wavefront calls it as often)
    int calls = 0;
    const auto over_waves = [&](int mine) __attribute__((always_inline)) -> int {
        if (WAVES == 1)
            return mine;
        int* const at = counts[calls & 1];
        ++calls;
        if (lane == 0)
            at[w] = mine;
        __syncthreads();
        return __builtin_amdgcn_readfirstlane((int)over_row((lane & 15) < WAVES ? (unsigned)at[lane % WAVES] : 0u, [](unsigned x, unsigned y) { return x + y; }));
    };
    const int groups = min(max((middle - t0 + 63) / 64, 0), V);  // of 64 tokens that have any to choose from
    const auto count = [&](unsigned least) __attribute__((always_inline)) -> int {
        int sum = 0;
#pragma unroll
        for (int v0 = 0; v0 < V; v0 += 4)
            if (v0 < groups) {
#pragma unroll
                for (int v = v0; v < v0 + 4; ++v)
                    sum += __popcll(__ballot(key[v] >= least));
            }
        return over_waves(sum);
    };
    unsigned floor = ~0u;  // keys from here on stay (no key is that large), and `ties` of those one below it where they are not all wanted
    int ties = 0;
    if (a.c > 0) {
        lowest = over_wave(lowest, [](unsigned x, unsigned y) { return min(x, y); });
        highest = over_wave(highest, [](unsigned x, unsigned y) { return max(x, y); });
        if (kBits) {
            int4* const own = (int4*)hist[local];
            for (int i = threadIdx.x % (64 * WAVES); i < kPlaces / 4; i += 64 * WAVES)
                own[i] = make_int4(0, 0, 0, 0);
            if (WAVES > 1 && threadIdx.x == 0)
                num_few = 0;
        }
        if (WAVES > 1) {
            __shared__ unsigned ends[2][WAVES];
            if (lane == 0) {
                ends[0][w] = lowest;
                ends[1][w] = highest;
            }
            __syncthreads();
            lowest = over_row(ends[0][lane % WAVES], [](unsigned x, unsigned y) { return min(x, y); });
            highest = over_row(ends[1][lane % WAVES], [](unsigned x, unsigned y) { return max(x, y); });
        }
        lowest = __builtin_amdgcn_readfirstlane(lowest);
        highest = __builtin_amdgcn_readfirstlane(highest);
        floor = lowest + 1u;
        int top = highest != floor ? 31 - __clz((int)(highest - floor)) : -1;
        bool exact = false;
        if (kBits && top >= kBits) {
            // the first kBits bits from a histogram, and the others of the few keys that share them with the c-th largest
            const int shift = top + 1 - kBits;
            int* const bins = hist[local];
#pragma unroll
            for (int v0 = 0; v0 < V; v0 += 4)
                if (v0 < groups) {
#pragma unroll
                    for (int v = v0; v < v0 + 4; ++v)
                        atomicAdd(&bins[key[v] ? place((int)((key[v] - floor) >> shift)) : kBins + 64 + lane], 1);  // (no token: a bin behind, of the lane's own)
                }
            if (WAVES > 1)
                __syncthreads();
            else
                wave_sync();
            // the bin of the c-th largest, how many lie above it and in it
            int bin = 0, above = 0, inside = 0;
            if (w == 0) {
                int here = 0;
#pragma unroll
                for (int i = 0; i < kOwn; ++i)
                    here += bins[place(lane * kOwn + i)];
                int from = here;  // keys of this lane's bins and of those above
#pragma unroll
                for (int o = 1; o < 64; o <<= 1) {
                    const int y = __shfl_down(from, o);
                    from += lane + o < 64 ? y : 0;
                }
                const int owner = 63 - __clzll((long long)__ballot(from >= a.c));
                const int over = __builtin_amdgcn_readlane(from - here, owner);
                // the owner's bins, a lane each, from the last one down
                const int mine = lane < kOwn ? bins[place(owner * kOwn + kOwn - 1 - lane)] : 0;
                int upto = mine;
#pragma unroll
                for (int o = 1; o < kOwn; o <<= 1) {
                    const int y = __shfl_up(upto, o);
                    upto += lane >= o ? y : 0;
                }
                const int at = __ffsll((unsigned long long)__ballot(lane < kOwn && over + upto >= a.c)) - 1;
                bin = owner * kOwn + kOwn - 1 - at;
                inside = __builtin_amdgcn_readlane(mine, at);
                above = over + __builtin_amdgcn_readlane(upto - mine, at);
            }
            if (WAVES > 1) {
                __shared__ int chosen[3];
                if (threadIdx.x == 0) {
                    chosen[0] = bin;
                    chosen[1] = above;
                    chosen[2] = inside;
                }
                __syncthreads();
                bin = __builtin_amdgcn_readfirstlane(chosen[0]);
                above = __builtin_amdgcn_readfirstlane(chosen[1]);
                inside = __builtin_amdgcn_readfirstlane(chosen[2]);
            }
            floor += (unsigned)bin << shift;
            exact = above + inside == a.c;
            top = shift - 1;
            if (!exact && inside <= 64) {
                int listed = 0;
#pragma unroll
                for (int v0 = 0; v0 < V; v0 += 4)
                    if (v0 < groups) {
#pragma unroll
                        for (int v = v0; v < v0 + 4; ++v) {
                            const bool hit = (key[v] - floor) >> shift == 0u;
                            if (WAVES > 1) {
                                if (hit)
                                    few[local][atomicAdd(&num_few, 1)] = key[v];
                                continue;
                            }
                            const unsigned long long some = __ballot(hit);
                            if (some != 0ull) {
                                if (hit)
                                    few[local][listed + lanes_below(some)] = key[v];
                                listed += __popcll(some);
                            }
                        }
                    }
                if (WAVES > 1)
                    __syncthreads();
                else
                    wave_sync();
                const unsigned mine = lane < inside ? few[local][lane] : 0u;
                for (int bit = top; bit >= 0 && !exact; --bit) {
                    const unsigned cand = floor + (1u << bit);
                    const int reach = cand > floor ? above + __popcll(__ballot(mine >= cand)) : 0;
                    if (reach >= a.c) {
                        floor = cand;
                        exact = reach == a.c;
                    }
                }
                top = -1;
            }
        }
        // (one more look at the end: how many lie above the c-th)
        for (int bit = top; bit >= -1 && !exact; --bit) {
            const unsigned cand = floor + (bit >= 0 ? 1u << bit : 1u);  // (below ~0: the largest key is +inf's)
            const int reach = count(cand);
            if (bit < 0) {
                floor = cand;
                ties = a.c - reach;
            } else if (cand > floor && reach >= a.c) {
                floor = cand;
                exact = reach == a.c;
            }
        }
    }
    // Which of tokens 64 v .. 64 v + 63 of this wavefront stay are 64 bits of lane v: all groups are counted at once, and loops walk those that
    // have something to do.
    const auto reach = [&](auto yes) __attribute__((always_inline)) -> unsigned long long {
        int lo = 0, hi = 0;
#pragma unroll
        for (int v0 = 0; v0 < V; v0 += 4)
            if (v0 < groups) {
#pragma unroll
                for (int v = v0; v < v0 + 4; ++v) {
                    const unsigned long long m = __ballot(yes(key[v]));
                    lo = lane == v ? (int)m : lo;
                    hi = lane == v ? (int)(m >> 32) : hi;
                }
            }
        return (unsigned long long)(unsigned)hi << 32 | (unsigned)lo;
    };
    const auto add = [](unsigned x, unsigned y) { return x + y; };
    // sum over the wavefronts in front of this one
    const auto in_front = [&](unsigned mine, int* at) __attribute__((always_inline)) -> unsigned {
        if (WAVES == 1)
            return 0u;
        if (lane == 0)
            at[w] = (int)mine;
        __syncthreads();
        return (unsigned)__builtin_amdgcn_readfirstlane((int)over_row(lane < w ? (unsigned)at[lane] : 0u, add));
    };
    unsigned long long kept = reach([&](unsigned k) { return k >= floor; });
    if (ties > 0) {  // the first `ties` of those that equal the c-th
        const unsigned long long equal = reach([&](unsigned k) { return k == floor - 1u; });
        const int here = __popcll(equal), upto = (int)up_to_lane((unsigned)here);
        const int wanted = ties - (int)in_front((unsigned)__builtin_amdgcn_readlane(upto, 31), sums[0]) - (upto - here);
        kept |= wanted >= here ? equal : 0ull;
        const unsigned long long part = __ballot(wanted > 0 && wanted < here);  // (a group at most)
        if (part != 0ull) {
            const int v = __ffsll(part) - 1, some = __builtin_amdgcn_readlane(wanted, v);
            const unsigned long long of = lane_bits(equal, v), first = __ballot((of >> lane & 1) && lanes_below(of) < some);
            kept |= lane == v ? first : 0ull;
        }
    }
    const int base = t0 + 64 * lane;
    const unsigned long long places = lane < V ? lowest_bits(early - base) : 0ull;
    kept |= lane < V ? lowest_bits(a.f - base) : 0ull;
    const unsigned long long gaps = ~kept & places, moves = kept & ~places;
    // (16 bits each: no more than half of the tokens move)
    const unsigned both = (unsigned)__popcll(gaps) << 16 | (unsigned)__popcll(moves), upto = up_to_lane(both);
    const unsigned before = upto - both + in_front((unsigned)__builtin_amdgcn_readlane((int)upto, 31), sums[1]);
    unsigned short* const list = moving[local];
    for (unsigned long long todo = __ballot(moves != 0ull); todo != 0ull; todo &= todo - 1ull) {
        const int v = __ffsll(todo) - 1;
        const unsigned long long some = lane_bits(moves, v);
        if (__builtin_amdgcn_inverse_ballot_w64(some))
            list[(__builtin_amdgcn_readlane((int)before, v) & 0xffff) + lanes_below(some)] = (unsigned short)(t0 + 64 * v + lane);
    }
    const auto fill = [&](int t, unsigned long long some, int at) __attribute__((always_inline)) {
        int from = t;
        if (__builtin_amdgcn_inverse_ballot_w64(some))
            from = (int)list[at + lanes_below(some)];
        if (t < early)
            source[t] = from;
    };
    if (WAVES == 1) {
        wave_sync();
#pragma unroll 4
        for (int v = 0; v < (early + 63) / 64; ++v)
            fill(64 * v + lane, lane_bits(gaps, v), (int)((unsigned)__builtin_amdgcn_readlane((int)before, v) >> 16));
    } else {
        // (by all wavefronts, not only those that have the early places)
        __shared__ unsigned long long gaps_of[WAVES == 1 ? 1 : WAVES * V];
        __shared__ unsigned before_of[WAVES == 1 ? 1 : WAVES * V];
        if (lane < V) {
            gaps_of[w * V + lane] = gaps;
            before_of[w * V + lane] = before >> 16;
        }
        __syncthreads();
#pragma unroll 2
        for (int v = w; v < (early + 63) / 64; v += WAVES) {
            const unsigned long long some = gaps_of[v];
            fill(64 * v + lane, (unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)(some >> 32)) << 32 |
                                    (unsigned)__builtin_amdgcn_readfirstlane((int)some),
                 __builtin_amdgcn_readfirstlane((int)before_of[v]));
        }
    }
    for (int i = threadIdx.x % (64 * WAVES); i < a.r; i += 64 * WAVES)
        source[early + i] = a.n - a.r + i;
}

// Places before this thread's for which `yes` holds, and their number over the workgroup.
__device__ __forceinline__ int before(bool yes, int* lds, int& all)
{
    const unsigned long long mine = __ballot(yes);
    const int wave = threadIdx.x >> 6;
    int count = __builtin_amdgcn_mbcnt_hi((unsigned)(mine >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mine, 0u));
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        lds[wave] = __popcll(mine);
    __syncthreads();
    all = 0;
    for (int w = 0; w < kLong / 64; ++w) {
        count += w < wave ? lds[w] : 0;
        all += lds[w];
    }
    return count;
}

// Rows of any length, from memory.
__global__ __launch_bounds__(kLong) void select_long(SelectParams p)
{
    __shared__ int hist[256], lds[kLong / 64], found[2];
    const int b = blockIdx.x / p.heads, j = blockIdx.x % p.heads, tid = threadIdx.x;
    const Row a = row_of(p, b);
    const int n = a.n, m = a.m, r = a.r, f = a.f, c = a.c;
    const float* const w = p.weights + (long long)blockIdx.x * p.stride;
    int* const source = p.source + (long long)blockIdx.x * p.source_stride;
    if (j == 0 && tid == 0)
        p.new_lens[b] = m;
    if (m == n) {
        for (int i = tid; i < m; i += kLong)
            source[i] = i;
        return;
    }
    // the c-th largest of tokens f .. n - r - 1: key `floor`, `ties` of which stay
    unsigned floor = 0u, mask = 0u;
    int ties = c;
    for (int shift = 24; shift >= 0 && c > 0; shift -= 8) {
        if (tid < 256)
            hist[tid] = 0;
        __syncthreads();
        for (int t = f + tid; t < n - r; t += kLong) {
            const unsigned key = key_of(w[t]);
            if ((key & mask) == floor)
                atomicAdd(&hist[key >> shift & 255u], 1);
        }
        __syncthreads();
        if (tid == 0) {
            int digit = 255, above = 0;
            while (above + hist[digit] < ties)
                above += hist[digit--];
            found[0] = digit;
            found[1] = above;
        }
        __syncthreads();
        floor |= (unsigned)found[0] << shift;
        mask |= 255u << shift;
        ties -= found[1];
    }
    // Places 0 .. m - r - 1 ("early"): tokens that stay, and gaps between them, which tokens m - r .. n - r - 1 that stay fill.  Both are
    // walked in ascending order, gaps and the tokens that fill them in step.
    __shared__ int gaps[kLong];
    const int early = m - r;
    int tied = 0;  // ties in front of the walk
    const auto stays = [&](int t, int end) {
        const unsigned key = t < end ? key_of(w[t]) : 0u;
        const bool middle = t >= f && t < end && c > 0, tie = middle && key == floor;
        int all;
        const int rank = tied + before(tie, lds, all);
        tied += all;
        return (t < f && t < end) || (middle && key > floor) || (tie && rank < ties);
    };
    for (int t0 = 0; t0 < early; t0 += kLong) {
        const int t = t0 + tid;
        const bool here = stays(t, early);
        if (t < early)
            source[t] = here ? t : -1;
    }
    __syncthreads();
    int listed = 0, used = 0, looked = 0;  // gaps in the list, those filled, and how far the places were looked through
    for (int t0 = early; t0 < n - r; t0 += kLong) {
        const int t = t0 + tid;
        const bool here = stays(t, n - r);
        int moving, done = 0;
        const int nth = before(here, lds, moving);
        while (done < moving) {
            if (used == listed) {
                listed = used = 0;
                while (listed == 0 && looked < early) {
                    const bool gap = looked + tid < early && source[looked + tid] < 0;
                    const int at = before(gap, lds, listed);
                    if (gap)
                        gaps[at] = looked + tid;
                    looked += kLong;
                }
                __syncthreads();
            }
            const int take = min(moving - done, listed - used);
            if (take <= 0)
                break;  // (there are as many gaps as tokens that fill them)
            if (here && nth >= done && nth < done + take)
                source[gaps[used + nth - done]] = t;
            __syncthreads();
            used += take;
            done += take;
        }
    }
    for (int i = early + tid; i < m; i += kLong)
        source[i] = n - m + i;
}

// A sequence's places in both tables: the first ones, and how many tokens they hold.
struct Places {
    int in0, out0;
    long long held, room;
};
__device__ __forceinline__ Places places_of(const CompactParams& p, int b)
{
    const int in0 = p.indptr[b], out0 = p.out_indptr[b], per = p.page_size ? 16 : 1;
    return {in0, out0, (long long)(p.indptr[b + 1] - in0) * per, (long long)(p.out_indptr[b + 1] - out0) * per};
}

// Where token t of a sequence lies for KV head j, in 16-byte pieces; `first`: its place in the table.
__device__ __forceinline__ long long row_at(const CompactParams& p, const int* pages, int first, int j, int t)
{
    return p.page_size ? (((long long)pages[first + (t >> 4)] * p.Hkv + j) * 16 + (t & 15)) * p.head_u4
                       : (long long)(first + t) * p.stride_u4 + (long long)j * p.head_u4;
}

// Weights, and the lengths: a workgroup a (sequence, KV head).
__device__ __forceinline__ void compact_weights(const CompactParams& p, int pair)
{
    constexpr int kEach = 4;
    const int j = pair % p.Hkv, b = pair / p.Hkv, tid = threadIdx.x;
    // (places and sources past their tables stay as they are; a source past the row of weights weighs 0.  All read at once, ahead of the first store)
    const int new_len = p.new_lens[b];
    const Places at = places_of(p, b);
    const int m = max(min(new_len, p.max_new), 0);
    if (j == 0 && tid == 0 && p.lens_out)
        p.lens_out[b] = m;
    if (!p.weights)
        return;
    const int* const source = p.source + b * p.seq_stride + j * p.head_stride;
    const int last = (int)min(at.room, (long long)m), stride = (int)p.weights_stride;
    const int held = (int)min(at.held, (long long)stride);
    const float* const w = p.weights + (long long)pair * p.weights_stride;
    float* const out = p.weights_out + (long long)pair * p.weights_stride;
    for (int i0 = 0; i0 < last; i0 += kEach * kThreads) {
        int src[kEach];
        float x[kEach];
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int i = i0 + e * kThreads + tid;
            src[e] = source[min(i, last - 1)];
        }
        // (what is not asked for reads another place: no branch, and all loads at once)
#pragma unroll
        for (int e = 0; e < kEach; ++e)
            x[e] = w[min(max(src[e], 0), stride - 1)];
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int i = i0 + e * kThreads + tid;
            if (i < last && src[e] >= i && (src[e] < held || src[e] >= stride))
                out[i] = src[e] < stride ? x[e] : 0.f;
        }
    }
    __syncthreads();
    for (long long i = m + tid; i < p.weights_stride; i += kThreads)
        out[i] = 0.f;
}

// Keys and values.  A workgroup takes pieces seg * width .. of the rows of one (sequence, KV head): of K and V, or of one of them
// (KINDS 2), and of all places, or (chunk > 0) of `chunk` of them; the workgroups from weights_from on move the weights.
template <int KINDS> __global__ __launch_bounds__(kThreads) void compact_rows(CompactParams p, int segs, int width, int chunk, int weights_from)
{
    if ((int)blockIdx.x >= weights_from) {
        compact_weights(p, (int)blockIdx.x - weights_from);
        return;
    }
    constexpr int kEach = KINDS == 1 ? 4 : 8;  // rows a thread has under way
    constexpr int kPlaces = 4 * kThreads;  // looked at in one go
    __shared__ long long from_at[kPlaces], to_at[kPlaces];
    __shared__ int lds[kThreads / 64];
    __shared__ int below;
    int rest = blockIdx.x;
    const int kind = rest % KINDS;
    rest /= KINDS;
    const int seg = rest % segs;
    rest /= segs;
    const int j = rest % p.Hkv;
    rest /= p.Hkv;
    const int b = rest % p.B, first = rest / p.B * chunk, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int m = max(min(p.new_lens[b], p.max_new), 0);
    int last = chunk > 0 ? min(m, first + chunk) : m;
    if (first >= last)
        return;
    const int* const source = p.source + b * p.seq_stride + j * p.head_stride;
    const auto [in0, out0, held, room] = places_of(p, b);
    const u32x4* const k = (const u32x4*)(kind == 1 ? p.v : p.k);
    u32x4* const k_out = (u32x4*)(kind == 1 ? p.v_out : p.k_out);
    const u32x4* const v = (const u32x4*)p.v;
    u32x4* const v_out = (u32x4*)p.v_out;
    const int rows = kThreads / width, mine = tid / width, piece = seg * width + tid % width;  // rows at a time, this thread's and its piece
    // whether anything is read from a place that is written: then one workgroup takes all places, and reads every group of them before
    // it writes them
    bool ordered = false;
    if (p.in_place) {
        if (tid == 0)
            below = 0;
        __syncthreads();
        bool any = false;
#pragma unroll 4
        for (int i = tid; i < m; i += kThreads) {
            const int src = source[i];
            any |= src > i && src < m;
        }
        if (__any(any) && lane == 0)
            below = 1;
        __syncthreads();
        ordered = below != 0;
        if (ordered && chunk > 0) {
            if (first > 0)
                return;
            last = m;
        }
    }
    for (int i0 = first; i0 < last; i0 += kPlaces) {
        // the places that get another token, listed in ascending order: a thread looks at kPlaces / kThreads in a row
        constexpr int kOwn = kPlaces / kThreads;
        int src[kOwn], mine_moves = 0;
        bool moves[kOwn];
#pragma unroll
        for (int o = 0; o < kOwn; ++o) {
            const int i = i0 + tid * kOwn + o;
            src[o] = i < last ? source[i] : -1;
        }
#pragma unroll
        for (int o = 0; o < kOwn; ++o) {
            const int i = i0 + tid * kOwn + o;
            moves[o] = src[o] >= i && src[o] < held && i < room && !(p.in_place && src[o] == i);
            mine_moves += moves[o];
        }
        int upto = mine_moves;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(upto, o);
            upto += lane >= o ? y : 0;
        }
        if (lane == 63)
            lds[wave] = upto;
        __syncthreads();
        int at = upto - mine_moves, all = 0;
#pragma unroll
        for (int w = 0; w < kThreads / 64; ++w) {
            at += w < wave ? lds[w] : 0;
            all += lds[w];
        }
#pragma unroll
        for (int o = 0; o < kOwn; ++o)
            if (moves[o]) {
                from_at[at] = row_at(p, p.pages, in0, j, src[o]);
                to_at[at] = row_at(p, p.out_pages, out0, j, i0 + tid * kOwn + o);
                ++at;
            }
        __syncthreads();
        for (int e0 = 0; e0 < all; e0 += kEach * rows) {
            u32x4 x[kEach], y[kEach];
            // (what has no row of its own repeats the last one)
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                const long long at_from = from_at[min(e0 + e * rows + mine, all - 1)] + piece;
                x[e] = k[at_from];
                if (KINDS == 1)
                    y[e] = v[at_from];
            }
            if (ordered) {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                __syncthreads();
            }
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                const int row = e0 + e * rows + mine;
                if (mine < rows && row < all) {
                    k_out[to_at[row] + piece] = x[e];
                    if (KINDS == 1)
                        v_out[to_at[row] + piece] = y[e];
                }
            }
        }
        __syncthreads();
    }
}

}  // namespace

hipError_t launch_select_kv(const SelectParams& p, hipStream_t s)
{
    const long long rows = p.seqs * p.heads;
#define SPD_SELECT(WAVES, V, ROWS) \
    hipLaunchKernelGGL((select_rows<WAVES, V, ROWS>), dim3((unsigned)((rows + ROWS - 1) / ROWS)), dim3(64 * WAVES * ROWS), 0, s, p)
    if (p.max_len <= 256) {
        SPD_SELECT(1, 4, 4);
    } else if (p.max_len <= 512) {
        SPD_SELECT(1, 8, 4);
    } else if (p.max_len <= 1024) {
        SPD_SELECT(1, 16, 4);
    } else if (p.max_len <= 2048) {
        SPD_SELECT(1, 32, 4);
    } else if (p.max_len <= 4096) {
        SPD_SELECT(4, 16, 1);
    } else if (p.max_len <= 8192) {
        SPD_SELECT(8, 16, 1);
    } else if (p.max_len <= 16384) {
        SPD_SELECT(16, 16, 1);
    } else if (p.max_len <= 32768) {
        SPD_SELECT(16, 32, 1);
    } else {
        hipLaunchKernelGGL(select_long, dim3((unsigned)rows), dim3(kLong), 0, s, p);
    }
#undef SPD_SELECT
    return hipGetLastError();
}

hipError_t launch_compact_kv(const CompactParams& p, hipStream_t s)
{
    const int pairs = p.B * p.Hkv;
    int kinds = 1, segs = 1, chunk = 0, chunks = 1;
    if (p.in_place) {
        // few rows: K and V, stretches of places, and where there are still few the pieces of a row, each have a workgroup.  Every one
        // looks through its row's list first: 512 rows of 2032 places of which few move 14.4 us, in twice as many workgroups 19.8, in one a row and kind 14.1.
        if (pairs < 1024) {
            kinds = 2;
            chunk = 256;
            while (chunk < (1 << 30) && (long long)pairs * kinds * ((p.max_new + chunk - 1) / chunk) > 2048)
                chunk *= 2;
            chunks = (p.max_new + chunk - 1) / chunk;
            while (p.head_u4 % (2 * segs) == 0 && 2 * segs * kinds * pairs * chunks <= 1024)
                segs *= 2;
        }
    } else {
        // a stretch is one trip of loads and stores (in stretches of 64, K and V together 7 % more)
        kinds = 2;
        chunk = 128;
        while (chunk < (1 << 30) && (long long)pairs * ((p.max_new + chunk - 1) / chunk) > 16384)
            chunk *= 2;
        chunks = (p.max_new + chunk - 1) / chunk;
    }
    const int copies = p.max_new > 0 ? pairs * kinds * segs * chunks : 0, others = p.weights || p.lens_out ? pairs : 0;
    if (copies + others == 0)
        return hipSuccess;
    if (kinds == 1)
        hipLaunchKernelGGL(compact_rows<1>, dim3((unsigned)(copies + others)), dim3(kThreads), 0, s, p, segs, p.head_u4 / segs, chunk, copies);
    else
        hipLaunchKernelGGL(compact_rows<2>, dim3((unsigned)(copies + others)), dim3(kThreads), 0, s, p, segs, p.head_u4 / segs, chunk, copies);
    return hipGetLastError();
}

}  // namespace spd
