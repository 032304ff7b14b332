// Launch planning of prompt_attn: host arithmetic only (no HIP, no allocation), so that it can also be
// compiled and exercised on a machine without a GPU.
#pragma once

#include "../../include/spdecode.h"

#include <stddef.h>
#include <stdint.h>

namespace spd {
namespace plan {

struct PromptPlan {
    int tiles;         // upper bound on the row tiles of all prompts, one KV head
    int paired;        // all units run at once, two a CU
    int by_length;     // units in the order of the tokens that they see, across prompts
    int num_splits;    // most parts of a prompt's tokens
    int split_tokens;  // fewest tokens of a part (the device knows the lengths, and how many tokens make the parts few enough)
    size_t acc_bytes, ml_bytes;
};

constexpr int kPromptRows = 128;       // (token, head of the group) rows per workgroup
constexpr int kPromptPlaces = 512;     // workgroups that run at once
constexpr int kPromptMaxSplits = 64;
// Up to so many prompts, the units of all of them run in the order of their tokens, so that a launch ends with its shortest; with more,
// prompt by prompt, so that those that run together read the same K and V.  Prompt by prompt / by length: 2 x 4096 fp32 tokens of 16 heads
// of 64 channels 644 / 634 us; 32 and 8 bf16 heads of 64 channels, 3 x 500..4001 113.1 / 109.5, 3 x 2000 73.3 / 69.5, 24 x 300..1000 90.7 / 92.2;
// of 128, 4 x 1000..4000 271 / 265, 8 x 2048 323 / 327, 26 x 300..512 85.7 / 98.8.
constexpr int kPromptsByLength = 4;
// Fewest tokens of a part: a tile of fp32 takes two to eight us, one of bf16 less than one, and a part costs its rows' states.
// 256 tokens of 4 / 1 fp32 heads of 64 channels, at least 32 / 64 / 128 tokens: 13.7 / 15.5 / 20.3 us; 32 new tokens over 1024 of 32 / 8
// bf16 heads, at least 64 / 96 / 128: 15.2 / 15.1 / 15.9, over 2048 18.4 / 17.6 / 17.4, over 4096 24.1 / 23.9 / 20.1.
inline int prompt_min_tokens(const spd_prompt_desc* d) { return d->dtype == SPD_BF16 ? 128 : 32; }

inline int check_prompt_desc(const spd_prompt_desc* d, bool queries)
{
    if (!d || d->num_kv_heads <= 0 || d->head_dim <= 0 || d->num_prompts <= 0 || d->q_stride < 0 || d->kv_stride < 0)
        return SPD_EINVAL;
    if (queries && (d->num_q_heads <= 0 || d->num_q_heads % d->num_kv_heads != 0))
        return SPD_EINVAL;
    if (d->dtype != SPD_F32 && d->dtype != SPD_BF16)
        return SPD_EUNSUPPORTED;
    if (d->page_size != 0 && d->page_size != 16)
        return SPD_EUNSUPPORTED;
    if (d->head_dim > 256 || d->head_dim % 8 != 0 || d->num_kv_heads > 65536 || d->num_q_heads > 65536 ||
        d->q_stride > (1 << 24) || d->kv_stride > (1 << 24))
        return SPD_EUNSUPPORTED;
    const int per_piece = d->dtype == SPD_BF16 ? 8 : 4;  // elements of 16 bytes
    if (d->q_stride % per_piece != 0 || d->kv_stride % per_piece != 0)
        return SPD_EINVAL;
    if ((queries && d->q_stride != 0 && d->q_stride < (int64_t)d->num_q_heads * d->head_dim) ||
        (d->kv_stride != 0 && d->kv_stride < (int64_t)d->num_kv_heads * d->head_dim))
        return SPD_EINVAL;
    return SPD_OK;
}

inline int make_prompt_plan(const spd_prompt_desc* d, int64_t total, int64_t max_query, int64_t max_kv, PromptPlan* out)
{
    const int rc = check_prompt_desc(d, true);
    if (rc != SPD_OK)
        return rc;
    const int64_t most = 0x7fffffff;
    if (total < 0 || max_query < 0 || max_kv < 0)
        return SPD_EINVAL;
    // row and token numbers are 32-bit; so is the grid
    if (total > most / d->num_q_heads || max_query > (1ll << 30) || max_kv > (1ll << 30))
        return SPD_EUNSUPPORTED;
    const int64_t group = d->num_q_heads / d->num_kv_heads;
    // a prompt's last tile may be partly filled, and no prompt has more tiles than its longest
    const int64_t per_prompt = (max_query * group + kPromptRows - 1) / kPromptRows;
    int64_t tiles = total * group / kPromptRows + d->num_prompts;
    if (per_prompt <= tiles / d->num_prompts)
        tiles = per_prompt * d->num_prompts;
    // Where the tiles alone leave CUs idle, the tokens are cut into parts, which another launch joins.
    const int64_t units = tiles * d->num_kv_heads;
    int64_t tokens = max_kv;
    if (units > 0 && units <= kPromptPlaces / 2) {
        tokens = units * max_kv / (2 * kPromptPlaces);
        const int64_t least = max_kv / kPromptMaxSplits > prompt_min_tokens(d) ? max_kv / kPromptMaxSplits : prompt_min_tokens(d);
        tokens = tokens > least ? tokens : least;
    }
    tokens = (tokens + 31) / 32 * 32;
    int64_t splits = tokens > 0 ? (max_kv + tokens - 1) / tokens : 1;
    splits = splits > 1 ? splits : 1;
    if (units > (1ll << 23) / splits)  // a launch counts its threads in 32 bits
        return SPD_EUNSUPPORTED;
    out->tiles = (int)tiles;
    out->paired = splits == 1 && d->causal != 0 && units > kPromptPlaces / 2 && units <= kPromptPlaces;
    out->by_length = splits == 1 && d->causal != 0 && !out->paired && d->num_prompts > 1 && d->num_prompts <= kPromptsByLength;
    out->num_splits = (int)splits;
    out->split_tokens = (int)tokens;
    const size_t states = splits > 1 ? (size_t)total * d->num_q_heads * splits : 0;
    out->acc_bytes = (states * d->head_dim * 4 + 255) / 256 * 256;
    out->ml_bytes = states * 4 * sizeof(float);
    return SPD_OK;
}

// ---- accumulate_kv_weights --------------------------------------------------------------------------------

constexpr int kWeightsFewRows = 32;   // rows up to which a wavefront keeps them all and streams the keys
constexpr int kWeightsMaxSplits = 32;

inline int weights_tile_tokens(bool bf16) { return bf16 ? 256 : 128; }  // of a workgroup with many rows

inline int64_t least(int64_t a, int64_t b) { return a < b ? a : b; }

struct WeightsPlan {
    int splits;              // parts of a sequence's rows
    size_t part_bytes;       // their sums
    size_t most_part_bytes;  // those of any call with no larger bounds and no more sequences or queries
};

inline int make_weights_plan(const spd_prompt_desc* d, int64_t total, int64_t max_query, int64_t max_kv, WeightsPlan* out)
{
    const int rc = check_prompt_desc(d, true);
    if (rc != SPD_OK)
        return rc;
    if (total < 0 || max_query < 0 || max_kv < 0)
        return SPD_EINVAL;
    const int64_t numbers = 0x7fffffff, group = d->num_q_heads / d->num_kv_heads;
    // row, token and workgroup numbers are 32-bit
    if (total > numbers / d->num_q_heads || max_query > (1ll << 30) / group || max_kv > (1ll << 30))
        return SPD_EUNSUPPORTED;
    const int64_t pairs = (int64_t)d->num_prompts * d->num_kv_heads;
    if (pairs > (1ll << 22) / ((max_kv + 63) / 64 + 1))
        return SPD_EUNSUPPORTED;
    out->splits = 1;
    out->part_bytes = out->most_part_bytes = 0;
    const int64_t rows = max_query * group, tokens = weights_tile_tokens(d->dtype == SPD_BF16);
    if (rows <= kWeightsFewRows)
        return SPD_OK;
    // (fewer queries or tokens may be cut into more parts, but parts times tiles stay below 4096 in bf16 and 8192 in fp32: 2^20 sums either way)
    const int64_t most = least(rows / (d->dtype == SPD_BF16 ? 128 : 32), kWeightsMaxSplits);
    if (most > 1)
        out->most_part_bytes = (size_t)least(most * pairs * max_kv, 1ll << 20) * sizeof(float);
    // The rows are cut into parts, which another launch adds (3 us and more), where the tiles that there are (total_queries says how many
    // of the longest sequence's each has) leave CUs idle, and where parts of 1024 rows and more even out what causal tiles have to do.  A block of
    // 32 rows takes 0.5 us: parts of at least 4 of them where three quarters of the places are idle, else 20 (512 queries over 4096 more
    // tokens, 32 / 8 heads: 34.8 us, whole 43.8; 256 over 8192: two parts 25.7, whole 24.1).  In fp32 a block takes 1 to 4 us, and parts may be as short as one.
    // 4 sequences of 373 to 2642 tokens, 4 / 2 heads: 25.2 us, by the longest alone 30.3; 4 fp32 ones of 456 to 2914, 60.4 and 71.2.
    const int64_t units = pairs * ((max_kv + tokens - 1) / tokens);
    if (units > 0) {
        const int64_t every = d->num_prompts * max_query, there = total < every ? units * total / every : units;
        const int64_t live = there > units / 4 ? there : units / 4 + 1;  // (no more than a guess, and workspace is for all)
        const int64_t places = d->head_dim <= 128 ? 512 : 256;  // two workgroups a CU, or one
        const int64_t fill = d->dtype != SPD_BF16 ? least(2048 / live, rows / 32)
                             : 2 * live <= places ? least(places / live, rows / (4 * live <= places ? 128 : 640)) : 1;
        const int64_t even = least(4096 / units, rows / 1024);
        out->splits = (int)least(fill > even ? fill : even, kWeightsMaxSplits);
        out->splits = out->splits > 1 ? out->splits : 1;
    }
    if (out->splits > 1)
        out->part_bytes = (size_t)out->splits * pairs * max_kv * sizeof(float);
    return SPD_OK;
}

}  // namespace plan
}  // namespace spd
