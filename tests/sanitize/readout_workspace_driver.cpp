// The workspaces that the plans of token_logprobs and accumulate_kv_weights ask for, against the sizes that their queries give for larger calls.
#include "../../paper_2502_02534_amd/csrc/logprobs_plan.h"
#include "../../paper_2502_02534_amd/csrc/prompt_plan.h"

#include <cstdio>
#include <random>

using namespace spd::plan;

static std::mt19937_64 rng(1);
static long long upto(long long most) { return (long long)(rng() % (unsigned long long)(most + 1)); }
static long long spread(int bits) { return upto((1ll << upto(bits)) - 1) + 1; }

int main()
{
    long long parts = 0;
    for (int n = 0; n < 200000; ++n) {
        const long long rows = spread(12), vocab = spread(21);
        const int top = (int)upto(64 < vocab ? 64 : vocab);
        const size_t size = logprobs_workspace_of_any(rows, vocab, top);
        for (int i = 0; i < 5; ++i) {
            const long long r = upto(rows), v = upto(vocab - 1) + 1;
            const size_t need = logprobs_workspace(r, v, (int)upto(top));
            parts += need > 0;
            if (need > size) {
                std::printf("FAILED: logprobs %lld x %lld needs %zu of %zu\n", r, v, need, size);
                return 1;
            }
        }
    }
    for (int n = 0; n < 200000; ++n) {
        spd_prompt_desc d = {};
        d.dtype = upto(1) ? SPD_BF16 : SPD_F32;
        d.num_kv_heads = (int)spread(4);
        d.num_q_heads = d.num_kv_heads * (int)spread(7);
        d.head_dim = 8 * ((int)upto(31) + 1);
        d.num_prompts = (int)spread(10);
        const long long query = spread(15), kv = spread(18);
        WeightsPlan p;
        if (make_weights_plan(&d, 0, query, kv, &p) != SPD_OK)
            continue;
        const size_t size = p.most_part_bytes;
        for (int i = 0; i < 5; ++i) {
            spd_prompt_desc e = d;
            e.num_prompts = (int)upto(d.num_prompts - 1) + 1;
            const long long q = upto(query), k = upto(kv), total = upto(e.num_prompts * q);
            if (make_weights_plan(&e, upto(3) ? total : e.num_prompts * q, q, k, &p) != SPD_OK)
                continue;
            parts += p.part_bytes > 0;
            if (p.part_bytes > size || p.most_part_bytes > size || p.part_bytes > p.most_part_bytes) {
                std::printf("FAILED: weights need %zu of %zu\n", p.part_bytes, size);
                return 1;
            }
        }
    }
    if (parts < 10000) {
        std::printf("FAILED: %lld plans in parts\n", parts);
        return 1;
    }
    std::printf("ok: %lld plans in parts\n", parts);
    return 0;
}
