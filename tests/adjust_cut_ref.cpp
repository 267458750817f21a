// How adjusted logits are cut into workgroups: prints the stretch, the rows of a workgroup and the workgroups for each
//   bf16 B rows V
// read from stdin.
#include <cstdio>

#include "../paper_2609_21858_amd/csrc/psd_adjust_plan.hpp"

int main() {
    int bf16, B, R, V;
    while (std::scanf("%d %d %d %d", &bf16, &B, &R, &V) == 4) {
        const psd::AdjustCut c = psd::adjust_cut(B, R, V, bf16 != 0);
        std::printf("%d %d %ld\n", c.seg, c.per, c.wgs(B, R));
    }
}
