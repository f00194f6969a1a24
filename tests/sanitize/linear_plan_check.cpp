// Reads T, K and N, prints the workspace of a linear call and what its products' parts and the bias's sums really take: forward of bf16 and of
// 8-bit operands, dx, dW, bias; and n, splits and blocks a split of each product.
#include <cstdio>

#include "linear_plan.h"

int main()
{
    long long T;
    int K, N;
    while (std::scanf("%lld %d %d", &T, &K, &N) == 3) {
        std::printf("%zu", cobalt::linear_workspace(T, K, N));
        const int64_t product[4][3] = {{N, T, cobalt::deep_blocks(K, cobalt::kDeep)}, {N, T, cobalt::deep_blocks(K, cobalt::kDeepBytes)},
                                       {K, T, cobalt::deep_blocks(N, cobalt::kDeep)}, {K, N, cobalt::deep_blocks(T, cobalt::kDeep)}};
        for (const auto& p : product) {
            const cobalt::LinearPlan plan = cobalt::linear_plan(p[0], p[1], p[2]);
            const long long parts = plan.splits > 1 ? static_cast<long long>(plan.splits) * p[0] * p[1] * 4 : 0;
            std::printf(" %lld %lld %d %d %d", static_cast<long long>(p[2]), parts, plan.n, plan.splits, plan.per_split);
        }
        std::printf(" %lld\n", static_cast<long long>(cobalt::bias_parts(T, N)) * N * 4);
    }
    return 0;
}
