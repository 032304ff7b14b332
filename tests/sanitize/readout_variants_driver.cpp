// Prints the kernel that token_logprobs takes for each "rows vocab top" triple of its arguments: threads, stripes, slices.
#include "../../paper_2502_02534_amd/csrc/logprobs_plan.h"

#include <cstdio>
#include <cstdlib>

int main(int argc, char** argv)
{
    for (int i = 1; i + 2 < argc; i += 3) {
        const spd::plan::LogprobsPlan p = spd::plan::make_logprobs_plan(std::atoll(argv[i]), std::atoll(argv[i + 1]));
        std::printf("%d %d %d\n", p.threads, p.stripes, p.slices);
    }
    return 0;
}
