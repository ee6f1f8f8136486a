// Host-only: the W8A8 product's plan for each "M N K workspace" read from standard input, as "shape split workgroups_n workgroups_m", behind the table of
// shapes, one "kind mb nt wk depth" a line, and an empty line.  Built and read by tests/test_w8a8_kernels.py.
#include "../../paper_2505_15909_amd/csrc/rtn_w8a8_plan.h"
#include <stdio.h>

int main() {
    for (const rtn::W8A8Shape& k : rtn::kShapes) printf("%d %d %d %d %d\n", k.kind, k.mb, k.nt, k.wk, k.depth);
    printf("\n");
    long M, N, K, workspace;
    while (scanf("%ld %ld %ld %ld", &M, &N, &K, &workspace) == 4) {
        const rtn::W8A8Plan p = rtn::w8a8_plan(M, N, K, (size_t)workspace);
        printf("%d %d %ld %ld\n", p.shape, p.split, (long)p.XB, (long)p.YB);
    }
    return 0;
}
