// Prints which kernels a call takes: "plan max_len S H eight_bits" -> wavefronts and parts, "products B d F" -> whether the products of
// rt_paged_products.hip are the faster ones, and the tiles of their workgroups for n_out = 3 d, d, F, d, 2 d.
#include "rt_paged_index.h"

#include <cstdio>
#include <cstdlib>
#include <cstring>

using namespace rt;

int main(int argc, char **argv)
{
    int v[4] = {};
    for (int i = 0; i < 4 && i + 2 < argc; ++i) v[i] = atoi(argv[i + 2]);
    if (argc > 1 && !strcmp(argv[1], "plan")) {
        const SplitPlan p = split_plan(v[0], v[1], v[2], v[3] != 0);
        printf("%d %d\n", p.waves, p.n_splits);
        return 0;
    }
    if (argc > 1 && !strcmp(argv[1], "products")) {
        const int outs[5] = {3 * v[1], v[1], v[2], v[1], 2 * v[1]};
        printf("%d", paged_products_take(v[0], v[1]) ? 1 : 0);
        for (int n : outs) printf(" %d", paged_product_tiles(n, v[0]));
        printf("\n");
        return 0;
    }
    return 2;
}
