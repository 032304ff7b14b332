// C ABI of what a step's two softmaxes say: token log probabilities, attention weights of cached tokens, their
// selection and compaction.  Argument checks and launches.
#include "../../include/spdecode.h"
#include "logprobs_plan.h"
#include "prompt_plan.h"
#include "spd_internal.h"

#include <math.h>

namespace {

using namespace spd::plan;

inline bool misaligned(const void* p, size_t a) { return ((uintptr_t)p % a) != 0; }

constexpr int64_t kMostBlocks = 1ll << 22;  // workgroups of up to 1024 threads: a launch counts its threads in 32 bits

int check_logprobs(int64_t rows, int64_t vocab, int32_t num_top)
{
    if (rows < 0 || vocab <= 0 || num_top < 0 || num_top > vocab)
        return SPD_EINVAL;
    if (num_top > SPD_MAX_TOP_TOKENS || vocab > (1ll << 30) || rows > kMostBlocks / ((vocab + 16383) / 16384) - 8)
        return SPD_EUNSUPPORTED;
    return SPD_OK;
}

int check_select(int64_t seqs, int32_t heads, int64_t max_kv)
{
    if (seqs <= 0 || heads <= 0 || max_kv < 0)
        return SPD_EINVAL;
    if (max_kv > (1 << 24) || seqs > (kMostBlocks - 1) / heads)
        return SPD_EUNSUPPORTED;
    return SPD_OK;
}

}  // namespace

extern "C" {

size_t token_logprobs_workspace_size(int64_t rows, int64_t vocab, int32_t num_top)
{
    return check_logprobs(rows, vocab, num_top) == SPD_OK ? logprobs_workspace_of_any(rows, vocab, num_top) + 256 : 0;
}

int token_logprobs(const void* logits, int32_t logits_dtype, int64_t rows, int64_t vocab, int64_t row_stride,
                   const float* temperature, const int32_t* tokens, int32_t num_top, float* logprobs, int32_t* ranks,
                   float* entropy, float* lse, int32_t* top_tokens, float* top_logprobs, void* workspace,
                   size_t workspace_bytes, void* stream)
{
    const int rc = check_logprobs(rows, vocab, num_top);
    if (rc != SPD_OK)
        return rc;
    if (!logits || row_stride < vocab || ((logprobs || ranks) && !tokens))
        return SPD_EINVAL;
    if (logits_dtype != SPD_F32 && logits_dtype != SPD_BF16)
        return SPD_EUNSUPPORTED;
    if (misaligned(logits, logits_dtype == SPD_BF16 ? 2 : 4))
        return SPD_EINVAL;
    const void* four[] = {temperature, tokens, logprobs, ranks, entropy, lse, top_tokens, top_logprobs};
    for (const void* x : four)
        if (misaligned(x, 4))
            return SPD_EINVAL;
    if (rows == 0)
        return SPD_OK;
    const int32_t tops = top_tokens || top_logprobs ? num_top : 0;
    const size_t need = logprobs_workspace(rows, vocab, tops);
    if (need > 0 && (!workspace || misaligned(workspace, 256) || workspace_bytes < need))
        return SPD_EWORKSPACE;
    spd::LogprobsParams p;
    p.logits = logits;
    p.bf16 = logits_dtype == SPD_BF16;
    p.rows = rows;
    p.vocab = vocab;
    p.stride = row_stride;
    p.temperature = temperature;
    p.tokens = tokens;
    p.top = tops;
    p.logprobs = logprobs;
    p.ranks = ranks;
    p.entropy = entropy;
    p.lse = lse;
    p.top_tokens = top_tokens;
    p.top_logprobs = top_logprobs;
    p.workspace = workspace;
    return spd::launch_token_logprobs(p, (hipStream_t)stream) == hipSuccess ? SPD_OK : SPD_ELAUNCH;
}

size_t accumulate_kv_weights_workspace_size(const spd_prompt_desc* desc, int64_t total_queries, int64_t max_query_len,
                                            int64_t max_kv_len)
{
    WeightsPlan pl;
    if (make_weights_plan(desc, total_queries, max_query_len, max_kv_len, &pl) != SPD_OK)
        return 0;
    return pl.most_part_bytes + 256;
}

int accumulate_kv_weights(const spd_prompt_desc* desc, const void* q, const void* k, const int32_t* query_indptr,
                          const int32_t* kv_lens, const int32_t* kv_indptr, const int32_t* kv_page_indices, const float* lse,
                          int64_t total_queries, int64_t max_query_len, int64_t max_kv_len, float decay,
                          const float* weights, float* weights_out, int64_t weights_stride, void* workspace,
                          size_t workspace_bytes, void* stream)
{
    WeightsPlan pl;
    const int rc = make_weights_plan(desc, total_queries, max_query_len, max_kv_len, &pl);
    if (rc != SPD_OK)
        return rc;
    if (!q || !k || !query_indptr || !kv_lens || !kv_indptr || !lse || !weights_out || (desc->page_size != 0 && !kv_page_indices))
        return SPD_EINVAL;
    if (weights_stride < max_kv_len || weights_stride > (1ll << 31))
        return weights_stride < max_kv_len ? SPD_EINVAL : SPD_EUNSUPPORTED;
    if (misaligned(q, 16) || misaligned(k, 16))
        return SPD_EINVAL;
    const void* four[] = {query_indptr, kv_lens, kv_indptr, kv_page_indices, lse, weights, weights_out};
    for (const void* x : four)
        if (misaligned(x, 4))
            return SPD_EINVAL;
    if (pl.splits > 1 && (!workspace || misaligned(workspace, 256) || workspace_bytes < pl.part_bytes))
        return SPD_EWORKSPACE;
    if (max_kv_len == 0)
        return SPD_OK;
    spd::KvWeightsParams p;
    p.dtype = desc->dtype;
    p.Hq = desc->num_q_heads;
    p.Hkv = desc->num_kv_heads;
    p.D = desc->head_dim;
    p.G = p.Hq / p.Hkv;
    p.B = desc->num_prompts;
    p.page_size = desc->page_size;
    p.causal = desc->causal != 0;
    const double scale = (desc->sm_scale > 0.f ? (double)desc->sm_scale : 1.0 / sqrt((double)p.D)) * 1.4426950408889634;
    p.scale_log2 = (float)scale;
    p.scale_rest = (float)(scale - (double)p.scale_log2);
    p.q = q;
    p.k = k;
    p.q_stride = desc->q_stride != 0 ? desc->q_stride : (long long)p.Hq * p.D;
    p.kv_stride = desc->kv_stride != 0 ? desc->kv_stride : (long long)p.Hkv * p.D;
    p.query_indptr = query_indptr;
    p.kv_lens = kv_lens;
    p.kv_indptr = kv_indptr;
    p.pages = kv_page_indices;
    p.lse = lse;
    p.max_query = (int)max_query_len;
    p.max_kv = (int)max_kv_len;
    p.decay = decay;
    p.weights = decay != 0.f ? weights : nullptr;
    p.weights_out = weights_out;
    p.stride = weights_stride;
    p.splits = pl.splits;
    p.part = (float*)workspace;
    return spd::launch_kv_weights(p, (hipStream_t)stream) == hipSuccess ? SPD_OK : SPD_ELAUNCH;
}

size_t select_kv_tokens_workspace_size(int64_t num_seqs, int32_t num_heads, int64_t max_kv_len)
{
    if (check_select(num_seqs, num_heads, max_kv_len) != SPD_OK)
        return 0;
    return 256;
}

int select_kv_tokens(const float* weights, int64_t weights_stride, int64_t num_seqs, int32_t num_heads, const int32_t* kv_lens,
                     int64_t max_kv_len, const int32_t* budgets, int64_t max_new_len, int32_t sinks, int32_t recent,
                     int32_t* source, int64_t source_stride, int32_t* new_lens, void* workspace, size_t workspace_bytes,
                     void* stream)
{
    const int rc = check_select(num_seqs, num_heads, max_kv_len);
    if (rc != SPD_OK)
        return rc;
    if (!weights || !kv_lens || !source || !new_lens || max_new_len < 0 || sinks < 0 || recent < 0)
        return SPD_EINVAL;
    if (new_lens == kv_lens)  // (written by a sequence's first head, read by all)
        return SPD_EINVAL;
    if (max_new_len > max_kv_len)
        max_new_len = max_kv_len;
    if (weights_stride < max_kv_len || source_stride < max_new_len)
        return SPD_EINVAL;
    const void* four[] = {weights, kv_lens, budgets, source, new_lens};
    for (const void* x : four)
        if (misaligned(x, 4))
            return SPD_EINVAL;
    (void)workspace;
    (void)workspace_bytes;
    spd::SelectParams p;
    p.weights = weights;
    p.stride = weights_stride;
    p.seqs = num_seqs;
    p.heads = num_heads;
    p.lens = kv_lens;
    p.max_len = (int)max_kv_len;
    p.budgets = budgets;
    p.max_new = (int)max_new_len;
    p.sinks = sinks;
    p.recent = recent;
    p.source = source;
    p.source_stride = source_stride;
    p.new_lens = new_lens;
    return spd::launch_select_kv(p, (hipStream_t)stream) == hipSuccess ? SPD_OK : SPD_ELAUNCH;
}

int compact_kv(const spd_prompt_desc* desc, const int32_t* source, int64_t source_seq_stride, int64_t source_head_stride,
               const int32_t* new_lens, int64_t max_new_len, const int32_t* kv_indptr, const int32_t* kv_page_indices,
               const void* k, const void* v, const int32_t* out_indptr, const int32_t* out_page_indices, void* k_out,
               void* v_out, const float* weights, float* weights_out, int64_t weights_stride, int32_t* lens_out, void* stream)
{
    const int rc = check_prompt_desc(desc, false);
    if (rc != SPD_OK)
        return rc;
    if (!source || !new_lens || !kv_indptr || !out_indptr || !k || !v || !k_out || !v_out || max_new_len < 0 ||
        source_seq_stride < 0 || source_head_stride < 0 || (weights != nullptr) != (weights_out != nullptr) ||
        (desc->page_size != 0 && (!kv_page_indices || !out_page_indices)))
        return SPD_EINVAL;
    if (weights && weights_stride < max_new_len)
        return SPD_EINVAL;
    // one list for all heads or all sequences, or lists that do not overlap
    if ((source_head_stride != 0 && source_head_stride < max_new_len) || (source_seq_stride != 0 && source_seq_stride < max_new_len))
        return SPD_EINVAL;
    if (max_new_len > (1ll << 30) || weights_stride > (1ll << 30) ||
        (int64_t)desc->num_prompts * desc->num_kv_heads > SPD_MAX_COMPACT_ROWS)
        return SPD_EUNSUPPORTED;
    const void* pools[] = {k, v, k_out, v_out};
    for (const void* x : pools)
        if (misaligned(x, 16))
            return SPD_EINVAL;
    const void* four[] = {source, new_lens, kv_indptr, kv_page_indices, out_indptr, out_page_indices, weights, weights_out, lens_out};
    for (const void* x : four)
        if (misaligned(x, 4))
            return SPD_EINVAL;
    // In place all of it, or none: what would be half of either cannot be what the caller wants.
    const bool same_k = k == k_out, same_v = v == v_out;
    const bool same_table = kv_indptr == out_indptr && (desc->page_size == 0 || kv_page_indices == out_page_indices);
    if (k_out == v_out || (same_table && same_k != same_v))
        return SPD_EINVAL;
    spd::CompactParams p;
    p.source = source;
    p.seq_stride = source_seq_stride;
    p.head_stride = source_head_stride;
    p.new_lens = new_lens;
    p.max_new = (int)max_new_len;
    p.B = desc->num_prompts;
    p.Hkv = desc->num_kv_heads;
    const int elt = desc->dtype == SPD_BF16 ? 2 : 4;
    p.head_u4 = desc->head_dim * elt / 16;
    p.page_size = desc->page_size;
    p.stride_u4 = desc->kv_stride != 0 ? desc->kv_stride * elt / 16 : (long long)p.Hkv * p.head_u4;
    p.indptr = kv_indptr;
    p.pages = kv_page_indices;
    p.k = k;
    p.v = v;
    p.out_indptr = out_indptr;
    p.out_pages = out_page_indices;
    p.k_out = k_out;
    p.v_out = v_out;
    p.weights = weights;
    p.weights_out = weights_out;
    p.weights_stride = weights_stride;
    p.lens_out = lens_out;
    p.in_place = same_table && same_k;
    return spd::launch_compact_kv(p, (hipStream_t)stream) == hipSuccess ? SPD_OK : SPD_ELAUNCH;
}

}  // extern "C"
