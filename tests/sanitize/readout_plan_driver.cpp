// Exercises the launch planners of token_logprobs and accumulate_kv_weights (host arithmetic, logprobs_plan.h and prompt_plan.h of
// paper_2502_02534_amd/csrc) under AddressSanitizer and UndefinedBehaviorSanitizer, and checks what the kernels rely on.
#include "../../paper_2502_02534_amd/csrc/logprobs_plan.h"
#include "../../paper_2502_02534_amd/csrc/prompt_plan.h"

#include <cstdio>
#include <initializer_list>

using namespace spd::plan;

static int fail(const char* what, long long a, long long b)
{
    std::printf("FAILED: %s (%lld, %lld)\n", what, a, b);
    return 1;
}

static int logprobs()
{
    long long cut = 0;
    for (long long rows : {0ll, 1ll, 2ll, 16ll, 64ll, 128ll, 129ll, 1024ll, 100000ll})
        for (long long vocab : {1ll, 7ll, 1024ll, 8192ll, 8193ll, 16383ll, 16384ll, 32767ll, 32768ll, 50257ll, 128256ll, 131064ll, 131065ll,
                                131072ll, 262144ll, 1ll << 20, (1ll << 30) - 1, 1ll << 30}) {
            const LogprobsPlan p = make_logprobs_plan(rows, vocab);
            if (p.slices < 1 || p.slice < 1 || p.slice % kChunk != 0 || p.slice > kMostSlice)
                return fail("slice", p.slice, p.slices);
            if ((long long)p.slice * p.slices < vocab || (long long)p.slice * (p.slices - 1) >= vocab)
                return fail("slices cover the vocabulary, and none is empty", p.slice, vocab);
            // a slice that starts within 16 bytes has up to seven places in front of it
            const int chunks = (p.slice + 2 * kChunk - 2) / kChunk, most = p.threads == 256 ? 256 * 8 : 512 * 32;
            if ((p.threads != 256 && p.threads != 512) || chunks > most)
                return fail("chunks of a workgroup", chunks, p.threads);
            if (logprobs_workspace(rows, vocab, 20) != (p.slices > 1 ? (size_t)rows * p.slices * (sizeof(spd::LogprobsPart) + 160) : 0))
                return fail("workspace", rows, vocab);
            cut += p.slices > 1;
        }
    return cut > 10 ? 0 : fail("plans with slices", cut, 10);
}

int main()
{
    if (logprobs() != 0)
        return 1;
    long long plans = 0, cut = 0, refused = 0;
    for (int dtype : {SPD_BF16, SPD_F32})
        for (int hkv : {1, 2, 8, 65536})
            for (int group : {1, 4, 7, 64})
                for (int dim : {8, 64, 80, 256})
                    for (int seqs : {1, 3, 64, 1000, 65536, 0x7fffffff})
                        for (long long total : {0ll, 1ll, 5000ll, 1ll << 20, 0x7fffffffll, 1ll << 40})
                            for (long long most : {0ll, 1ll, 8ll, 9ll, 128ll, 4097ll, 1ll << 30, 1ll << 62})
                                for (long long kv : {0ll, 1ll, 31ll, 200ll, 8192ll, 16384ll, 1ll << 30, 1ll << 62}) {
                                    spd_prompt_desc d = {};
                                    d.dtype = dtype, d.num_kv_heads = hkv, d.num_q_heads = hkv > 100 ? hkv : hkv * group, d.head_dim = dim;
                                    d.num_prompts = seqs;
                                    WeightsPlan p;
                                    if (make_weights_plan(&d, total, most, kv, &p) != SPD_OK) {
                                        ++refused;
                                        continue;
                                    }
                                    ++plans;
                                    const long long g = d.num_q_heads / hkv, pairs = (long long)seqs * hkv, rows = most * g;
                                    if (rows > 1ll << 30)
                                        return fail("rows of 32 bits", rows, most);
                                    if (p.splits < 1 || p.splits > kWeightsMaxSplits)
                                        return fail("parts", p.splits, rows);
                                    const long long tokens = weights_tile_tokens(dtype == SPD_BF16), tiles = (kv + tokens - 1) / tokens;
                                    if (tiles * pairs * p.splits > 1ll << 22)
                                        return fail("grid", tiles * pairs, p.splits);
                                    if (pairs * ((kv + 15) / 16) > 0x7fffffffll / 4)
                                        return fail("grid of few rows", pairs, kv);
                                    if (p.splits > 1 && (rows <= kWeightsFewRows || pairs > 65535 || rows < 32ll * p.splits))
                                        return fail("parts that are not worth it, or a join's grid", pairs, p.splits);
                                    if (p.part_bytes != (p.splits > 1 ? (size_t)p.splits * pairs * kv * 4 : 0))
                                        return fail("workspace", (long long)p.part_bytes, pairs);
                                    cut += p.splits > 1;
                                }
    if (plans < 1000 || cut < 100 || refused < 1000)
        return fail("plans", plans, cut);
    std::printf("ok: %lld plans, %lld in parts, %lld refused\n", plans, cut, refused);
    return 0;
}
