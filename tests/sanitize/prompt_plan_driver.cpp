// Exercises the launch planner of prompt_attn (host arithmetic, paper_2502_02534_amd/csrc/prompt_plan.h) under
// AddressSanitizer and UndefinedBehaviorSanitizer over a grid of descriptions and bounds, and checks what the kernels rely on.
#include "../../paper_2502_02534_amd/csrc/prompt_plan.h"

#include <cstdio>
#include <initializer_list>

using namespace spd::plan;

static int fail(const char* what, long long a, long long b)
{
    std::printf("FAILED: %s (%lld, %lld)\n", what, a, b);
    return 1;
}

int main()
{
    long long plans = 0, cut = 0, pairs = 0, refused = 0;
    for (int dtype : {SPD_BF16, SPD_F32})
        for (int hkv : {1, 2, 8, 65536})
            for (int group : {1, 4, 7})
                for (int dim : {8, 64, 80, 256})
                    for (int prompts : {1, 3, 64, 1000, 0x7fffffff})
                        for (int causal : {0, 1})
                            for (long long total : {0ll, 1ll, 127ll, 129ll, 5000ll, 1ll << 20, 0x7fffffffll, 1ll << 40})
                                for (long long most : {1ll, 128ll, 4097ll, 1ll << 30, 1ll << 62})
                                    for (long long kv : {0ll, 1ll, 31ll, 200ll, 8192ll, 1ll << 30, 1ll << 62}) {
                                        spd_prompt_desc d = {};
                                        d.dtype = dtype, d.num_kv_heads = hkv, d.num_q_heads = hkv > 100 ? hkv : hkv * group, d.head_dim = dim;
                                        d.num_prompts = prompts, d.causal = causal;
                                        PromptPlan p;
                                        if (make_prompt_plan(&d, total, most, kv, &p) != SPD_OK) {
                                            ++refused;
                                            continue;
                                        }
                                        ++plans;
                                        const long long g = d.num_q_heads / hkv;
                                        // a tile per prompt may be partly filled: 128-row tiles of any division of the queries
                                        const long long need = total == 0 ? 0 : (total * g + kPromptRows - 1) / kPromptRows;
                                        const long long units = (long long)p.tiles * hkv;
                                        if (p.tiles < 0 || (most * prompts >= total && p.tiles < need))
                                            return fail("fewer tiles than rows", p.tiles, need);
                                        if (p.num_splits < 1 || p.num_splits > kPromptMaxSplits + 1)
                                            return fail("parts", p.num_splits, kv);
                                        if (units * p.num_splits > 1ll << 23)
                                            return fail("grid", units, p.num_splits);
                                        if ((long long)p.num_splits * p.split_tokens < kv || p.split_tokens % 32 != 0)
                                            return fail("parts do not cover the tokens", p.split_tokens, kv);
                                        if (p.num_splits > 1 && (units > kPromptPlaces / 2 || p.split_tokens < prompt_min_tokens(&d)))
                                            return fail("parts where the tiles are enough, or too short", units, p.split_tokens);
                                        if (p.paired && (p.num_splits > 1 || !causal || units <= kPromptPlaces / 2 || units > kPromptPlaces))
                                            return fail("pairs", units, p.num_splits);
                                        if (p.by_length && (p.num_splits > 1 || !causal || p.paired || prompts < 2 || prompts > 64))
                                            return fail("order", prompts, p.num_splits);
                                        const size_t states = p.num_splits > 1 ? (size_t)total * d.num_q_heads * p.num_splits : 0;
                                        if (p.ml_bytes != states * 16 || p.acc_bytes < states * dim * (dtype == SPD_BF16 ? 2 : 4) || p.acc_bytes % 256 != 0)
                                            return fail("workspace", (long long)p.acc_bytes, (long long)states);
                                        cut += p.num_splits > 1;
                                        pairs += p.paired;
                                    }
    if (cut == 0 || pairs == 0 || refused == 0)
        return fail("a kind of plan did not occur", cut, pairs);
    // the lines, from both sides: 256 | 257 units of one row tile, 512 | 513
    for (int units : {256, 257, 512, 513}) {
        spd_prompt_desc d = {};
        d.dtype = SPD_BF16, d.num_kv_heads = 1, d.num_q_heads = 1, d.head_dim = 64, d.num_prompts = units, d.causal = 1;
        PromptPlan p;
        if (make_prompt_plan(&d, units, 1, 4096, &p) != SPD_OK || p.tiles != units)
            return fail("tiles of single tokens", p.tiles, units);
        if ((p.num_splits > 1) != (units <= 256) || (p.paired != 0) != (units > 256 && units <= 512))
            return fail("line", units, p.num_splits);
    }
    std::printf("ok %lld plans, %lld in parts, %lld in pairs, %lld refused\n", plans, cut, pairs, refused);
    return 0;
}
