// Host-only: the W8A8 product's plan for each "M N K workspace" read from standard input, as "shape kind split workgroups_n workgroups_m".  Built and read by
// tests/test_w8a8_kernels.py.
#include "../../paper_2505_15909_amd/csrc/rtn_w8a8_plan.h"
#include <stdio.h>

int main() {
    long M, N, K, workspace;
    while (scanf("%ld %ld %ld %ld", &M, &N, &K, &workspace) == 4) {
        const rtn::W8A8Plan p = rtn::w8a8_plan(M, N, K, (size_t)workspace);
        printf("%d %d %d %ld %ld\n", p.shape, rtn::kShapes[p.shape].kind, p.split, (long)p.XB, (long)p.YB);
    }
    return 0;
}
