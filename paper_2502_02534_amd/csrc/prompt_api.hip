// C ABI of the operators around the decode step: prompt attention, page tables, KV writes, token marks and
// logit penalties.  Argument checks and launches.
#include "../../include/spdecode.h"
#include "prompt_plan.h"
#include "spd_internal.h"

#include <math.h>

namespace {

using namespace spd::plan;

inline bool misaligned(const void* p, size_t a) { return ((uintptr_t)p % a) != 0; }

constexpr int64_t kMostInt = 0x7fffffff;
constexpr int64_t kMostBlocks = 1ll << 22;  // workgroups of up to 1024 threads: a launch counts its threads in 32 bits

int page_tables(int64_t num_requests, int32_t page_size, const int32_t* lens, const int32_t* held_lens,
                const int32_t* held_indptr, const int32_t* held_pages, const int32_t* free_pages, int64_t num_free,
                const int32_t* free_begin, int64_t max_pages, int64_t max_tokens, int32_t* page_indptr,
                int32_t* page_indices, int32_t* lens_out, int32_t* new_indptr, int64_t* slot_map, int32_t* free_end,
                int32_t* packed_indptr, int32_t* packed_lens, void* workspace, size_t workspace_bytes, void* stream)
{
    if (num_requests <= 0 || num_free < 0 || max_pages < 0 || max_tokens < 0 || page_size < 1)
        return SPD_EINVAL;
    if (page_size > 65536 || num_requests >= kMostInt || num_free > kMostInt || max_pages > kMostInt || max_tokens > kMostInt)
        return SPD_EUNSUPPORTED;
    if (!lens || !page_indptr || !lens_out || !new_indptr || !free_end || (num_free > 0 && !free_pages) ||
        (max_pages > 0 && !page_indices))
        return SPD_EINVAL;
    if ((held_lens || held_indptr || held_pages) && (!held_lens || !held_indptr || !held_pages))
        return SPD_EINVAL;
    const void* ints[] = {lens, held_lens, held_indptr, held_pages, free_pages, free_begin, page_indptr, page_indices,
                          lens_out, new_indptr, free_end, packed_indptr, packed_lens};
    for (const void* x : ints)
        if (misaligned(x, 4))
            return SPD_EINVAL;
    if (misaligned(slot_map, 8) || free_begin == free_end)
        return SPD_EINVAL;
    if (!workspace || misaligned(workspace, 256) || workspace_bytes < build_page_tables_workspace_size(num_requests))
        return SPD_EWORKSPACE;
    spd::PageTableParams p;
    p.n = num_requests;
    p.page_size = page_size;
    p.lens = lens;
    p.held_lens = held_lens;
    p.held_indptr = held_indptr;
    p.held_pages = held_pages;
    p.free_pages = free_pages;
    p.num_free = num_free;
    p.free_begin = free_begin;
    p.max_pages = max_pages;
    p.max_tokens = max_tokens;
    p.page_indptr = page_indptr;
    p.page_indices = page_indices;
    p.lens_out = lens_out;
    p.new_indptr = new_indptr;
    p.slot_map = (long long*)slot_map;
    p.free_end = free_end;
    p.packed_indptr = packed_indptr;
    p.packed_lens = packed_lens;
    p.first_free = (int*)workspace;
    return spd::launch_page_tables(p, (hipStream_t)stream) == hipSuccess ? SPD_OK : SPD_ELAUNCH;
}

}  // namespace

extern "C" {

size_t prompt_attn_workspace_size(const spd_prompt_desc* desc, int64_t total_queries, int64_t max_query_len, int64_t max_kv_len)
{
    PromptPlan pl;
    if (make_prompt_plan(desc, total_queries, max_query_len, max_kv_len, &pl) != SPD_OK)
        return 0;
    return pl.acc_bytes + pl.ml_bytes + 256;
}

int prompt_attn(const spd_prompt_desc* desc, const void* q, const void* k, const void* v, const int32_t* query_indptr,
                const int32_t* kv_lens, const int32_t* kv_indptr, const int32_t* kv_page_indices, int64_t total_queries,
                int64_t max_query_len, int64_t max_kv_len, void* out, float* lse_out, void* workspace,
                size_t workspace_bytes, void* stream)
{
    PromptPlan pl;
    const int rc = make_prompt_plan(desc, total_queries, max_query_len, max_kv_len, &pl);
    if (rc != SPD_OK)
        return rc;
    if (!q || !k || !v || !query_indptr || !kv_lens || !kv_indptr || !out || (desc->page_size != 0 && !kv_page_indices))
        return SPD_EINVAL;
    if (misaligned(q, 16) || misaligned(k, 16) || misaligned(v, 16) || misaligned(out, 16))
        return SPD_EINVAL;
    if (misaligned(query_indptr, 4) || misaligned(kv_lens, 4) || misaligned(kv_indptr, 4) || misaligned(kv_page_indices, 4) ||
        misaligned(lse_out, 4))
        return SPD_EINVAL;
    if (pl.num_splits > 1 && (!workspace || misaligned(workspace, 256) || workspace_bytes < pl.acc_bytes + pl.ml_bytes))
        return SPD_EWORKSPACE;
    if (total_queries == 0 || pl.tiles == 0)
        return SPD_OK;
    spd::PromptParams p;
    p.dtype = desc->dtype;
    p.Hq = desc->num_q_heads;
    p.Hkv = desc->num_kv_heads;
    p.D = desc->head_dim;
    p.G = p.Hq / p.Hkv;
    p.B = desc->num_prompts;
    p.page_size = desc->page_size;
    p.causal = desc->causal != 0;
    const float scale = desc->sm_scale > 0.f ? desc->sm_scale : 1.f / sqrtf((float)p.D);
    p.scale_log2 = scale * spd::kLog2e;
    p.q = q;
    p.k = k;
    p.v = v;
    p.q_stride = desc->q_stride != 0 ? desc->q_stride : (long long)p.Hq * p.D;
    p.kv_stride = desc->kv_stride != 0 ? desc->kv_stride : (long long)p.Hkv * p.D;
    p.query_indptr = query_indptr;
    p.kv_lens = kv_lens;
    p.kv_indptr = kv_indptr;
    p.pages = kv_page_indices;
    p.tiles = pl.tiles;
    p.paired = pl.paired;
    p.by_length = pl.by_length;
    p.num_splits = pl.num_splits;
    p.split_tokens = pl.split_tokens;
    p.rows = total_queries * p.Hq;
    p.part_acc = workspace;
    p.part_ml = (float4*)((char*)workspace + pl.acc_bytes);
    p.out = out;
    p.lse = lse_out;
    return spd::launch_prompt_attn(p, (hipStream_t)stream) == hipSuccess ? SPD_OK : SPD_ELAUNCH;
}

size_t build_page_tables_workspace_size(int64_t num_requests)
{
    if (num_requests <= 0 || num_requests >= kMostInt)
        return 0;
    return ((size_t)num_requests * 4 + 255) / 256 * 256;
}

int build_page_tables(int64_t num_requests, int32_t page_size, const int32_t* lens, const int32_t* held_lens,
                      const int32_t* held_indptr, const int32_t* held_pages, const int32_t* free_pages, int64_t num_free,
                      const int32_t* free_begin, int64_t max_pages, int64_t max_tokens, int32_t* page_indptr,
                      int32_t* page_indices, int32_t* lens_out, int32_t* new_indptr, int64_t* slot_map, int32_t* free_end,
                      void* workspace, size_t workspace_bytes, void* stream)
{
    return page_tables(num_requests, page_size, lens, held_lens, held_indptr, held_pages, free_pages, num_free, free_begin, max_pages,
                       max_tokens, page_indptr, page_indices, lens_out, new_indptr, slot_map, free_end, nullptr, nullptr, workspace,
                       workspace_bytes, stream);
}

int build_page_tables_packed(int64_t num_requests, int32_t page_size, const int32_t* lens, const int32_t* held_lens,
                             const int32_t* held_indptr, const int32_t* held_pages, const int32_t* free_pages, int64_t num_free,
                             const int32_t* free_begin, int64_t max_pages, int64_t max_tokens, int32_t* page_indptr,
                             int32_t* page_indices, int32_t* lens_out, int32_t* new_indptr, int64_t* slot_map, int32_t* free_end,
                             int32_t* packed_indptr, int32_t* packed_lens, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!packed_indptr || !packed_lens)
        return SPD_EINVAL;
    return page_tables(num_requests, page_size, lens, held_lens, held_indptr, held_pages, free_pages, num_free, free_begin, max_pages,
                       max_tokens, page_indptr, page_indices, lens_out, new_indptr, slot_map, free_end, packed_indptr, packed_lens,
                       workspace, workspace_bytes, stream);
}

int write_prompt_kv(const spd_prompt_desc* desc, const void* k, const void* v, const int64_t* slot_map, int64_t num_tokens,
                    int64_t num_pages, void* k_pool, void* v_pool, void* stream)
{
    const int rc = check_prompt_desc(desc, false);
    if (rc != SPD_OK)
        return rc;
    if (num_tokens < 0 || num_pages < 0 || !k || !v || !slot_map || !k_pool || !v_pool)
        return SPD_EINVAL;
    if (misaligned(k, 16) || misaligned(v, 16) || misaligned(k_pool, 16) || misaligned(v_pool, 16) || misaligned(slot_map, 8))
        return SPD_EINVAL;
    if (num_tokens > (1ll << 30) || num_pages > (1ll << 40))
        return SPD_EUNSUPPORTED;
    if (num_tokens == 0 || num_pages == 0)
        return SPD_OK;
    const int elt = desc->dtype == SPD_BF16 ? 2 : 4;
    spd::KvWriteParams p;
    p.k = k;
    p.v = v;
    p.slots = (const long long*)slot_map;
    p.k_pool = k_pool;
    p.v_pool = v_pool;
    p.tokens = num_tokens;
    p.num_slots = num_pages * (desc->page_size != 0 ? desc->page_size : 1);
    p.Hkv = desc->num_kv_heads;
    p.head_u4 = desc->head_dim * elt / 16;
    p.stride_u4 = desc->kv_stride != 0 ? desc->kv_stride * elt / 16 : (long long)p.Hkv * p.head_u4;
    p.page_size = desc->page_size;
    if (num_tokens > 4 * kMostBlocks * 255 / ((long long)p.Hkv * p.head_u4))
        return SPD_EUNSUPPORTED;
    return spd::launch_kv_write(p, (hipStream_t)stream) == hipSuccess ? SPD_OK : SPD_ELAUNCH;
}

int mark_prompt_tokens(const int32_t* tokens, const int32_t* indptr, int64_t num_prompts, int64_t vocab, uint32_t* bits,
                       int64_t bits_stride, int32_t accumulate, void* stream)
{
    if (!tokens || !indptr || !bits || num_prompts <= 0 || vocab <= 0 || bits_stride < (vocab + 31) / 32)
        return SPD_EINVAL;
    if (misaligned(tokens, 4) || misaligned(indptr, 4) || misaligned(bits, 4))
        return SPD_EINVAL;
    if (vocab > (1 << 20) || num_prompts >= kMostBlocks)
        return SPD_EUNSUPPORTED;
    return spd::launch_mark_tokens(tokens, indptr, num_prompts, vocab, bits, bits_stride, accumulate != 0,
                                   (hipStream_t)stream) == hipSuccess ? SPD_OK : SPD_ELAUNCH;
}

int penalize_logits(const void* logits, int32_t logits_dtype, int64_t rows, int64_t vocab, int64_t row_stride,
                    const spd_penalties* pen, float* out, int64_t out_stride, void* stream)
{
    if (!logits || !pen || !out || rows < 0 || vocab <= 0 || row_stride < vocab || out_stride < vocab)
        return SPD_EINVAL;
    if (logits_dtype != SPD_F32 && logits_dtype != SPD_BF16)
        return SPD_EUNSUPPORTED;
    if (vocab > (1ll << 30) || rows > kMostBlocks / ((vocab + 16383) / 16384) - 8 || pen->max_tokens > (1ll << 24))
        return SPD_EUNSUPPORTED;
    if (misaligned(logits, logits_dtype == SPD_BF16 ? 2 : 4) || misaligned(out, 4))
        return SPD_EINVAL;
    if ((const void*)out == logits && (logits_dtype != SPD_F32 || row_stride != out_stride))
        return SPD_EINVAL;
    if (pen->tokens && (!pen->token_lens || pen->max_tokens < 0))
        return SPD_EINVAL;
    if (pen->bias_tokens && (!pen->bias_indptr || !pen->bias_values))
        return SPD_EINVAL;
    const int64_t words = (vocab + 31) / 32;
    if ((pen->prompt_bits && pen->prompt_bits_stride < words) || (pen->allowed_bits && pen->allowed_stride < words))
        return SPD_EINVAL;
    const void* four[] = {pen->repetition, pen->frequency, pen->presence, pen->prompt_bits, pen->prompt_of_row, pen->tokens,
                          pen->token_lens, pen->bias_indptr, pen->bias_tokens, pen->bias_values, pen->allowed_bits,
                          pen->allowed_of_row};
    for (const void* x : four)
        if (misaligned(x, 4))
            return SPD_EINVAL;
    if (rows == 0)
        return SPD_OK;
    spd::LogitsParams p;
    p.logits = logits;
    p.bf16 = logits_dtype == SPD_BF16;
    p.rows = rows;
    p.vocab = vocab;
    p.stride = row_stride;
    p.out_stride = out_stride;
    p.out = out;
    p.repetition = pen->repetition;
    p.frequency = pen->frequency;
    p.presence = pen->presence;
    p.prompt_bits = pen->prompt_bits;
    p.prompt_stride = pen->prompt_bits_stride;
    p.prompt_of_row = pen->prompt_of_row;
    p.tokens = pen->tokens;
    p.token_row_stride = pen->token_row_stride;
    p.token_step_stride = pen->token_step_stride;
    p.token_lens = pen->token_lens;
    p.bias_indptr = pen->bias_indptr;
    p.bias_tokens = pen->bias_tokens;
    p.bias_values = pen->bias_values;
    p.allowed_bits = pen->allowed_bits;
    p.allowed_stride = pen->allowed_stride;
    p.allowed_of_row = pen->allowed_of_row;
    p.max_tokens = (int)pen->max_tokens;
    return spd::launch_penalize_logits(p, (hipStream_t)stream) == hipSuccess ? SPD_OK : SPD_ELAUNCH;
}

}  // extern "C"
