// Reads "T features K qkv swiglu scratch" lines and prints how an int8 projection of that size runs (gemm_plan_i8; host arithmetic alone):
// path, tile rows (or the tile of linear_rows_kernel), k ranges, tiles in k ranges at the end, columns of the first launch of two.
#include <cstdio>

#include "relserve_internal.h"

int main() {
    int T, K, qkv, swiglu, scratch;
    long long features;
    while (std::scanf("%d %lld %d %d %d %d", &T, &features, &K, &qkv, &swiglu, &scratch) == 6) {
        const relserve::GemmPlanI8 p = relserve::gemm_plan_i8(T, features, K, qkv != 0, swiglu != 0, scratch != 0);
        std::printf("%d %d %d %d %d\n", p.path, p.rows, p.ranges, p.tail_tiles, p.cols1);
    }
    return 0;
}
