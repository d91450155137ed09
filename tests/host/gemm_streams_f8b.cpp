// Reads "T N K epilogue scratch" lines and prints how a block-scaled projection of that size runs (gemm_plan_f8b; host arithmetic alone): tile, k ranges,
// whether its weights go past the caches.
#include <cstdio>

#include "relserve_internal.h"

int main() {
    int T, N, K, epilogue, scratch;
    while (std::scanf("%d %d %d %d %d", &T, &N, &K, &epilogue, &scratch) == 5) {
        const relserve::GemmPlanF8b p = relserve::gemm_plan_f8b(T, N, K, epilogue, scratch != 0);
        std::printf("%d %d %d\n", p.tile, p.ranges, p.streamed);
    }
    return 0;
}
