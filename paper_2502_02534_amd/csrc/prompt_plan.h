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

}  // namespace plan
}  // namespace spd
