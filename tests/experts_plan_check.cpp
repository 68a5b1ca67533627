// Which kernel a product of experts, or a gradient, gets (sparq_mx_experts_plan.h), asked on the host.
//   experts_plan_check product M N K experts offsets function residual kept    prints "tile fragments parts"
//   experts_plan_check dx TYPE M N K experts | dw TYPE M N K experts           prints "tile"  (TYPE: 0 fp32, 1 fp16, 2 bf16)
#define __shared__
#include <stdio.h>
#include <stdlib.h>

#include "../paper_2105_11010_amd/csrc/sparq_mx_experts_plan.h"

using namespace sparq::mx;

void gpu::load(const Buffer&, uint32_t, uint32_t, int) {}

int main(int argc, char** argv) {
    std::vector<int64_t> n;
    for (int i = 0; i < argc; ++i) n.push_back(atoll(argv[i]));
    if (argc == 10 && !strcmp(argv[1], "product")) {
        const ExpertsPlan p = experts_plan(n[2], (int)n[3], (int)n[4], (int)n[5], n[6] != 0, (int)n[7], n[8] != 0, n[9] != 0);
        printf("%d %d %d\n", p.tile, p.fragments, p.parts);
    } else if (argc == 7 && !strcmp(argv[1], "dx")) {
        printf("%d\n", dx_tile((int)n[2], n[3], (int)n[5], (int)n[6]));
    } else if (argc == 7 && !strcmp(argv[1], "dw")) {
        printf("%d\n", dw_tile((int)n[2], n[3], (int)n[4], (int)n[5], (int)n[6]));
    } else {
        return 2;
    }
    return 0;
}
