// How linear's products are cut into tiles and parts of k, and the workspace that this takes (host only).
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace cobalt {

constexpr int kTileM = 256;              // i of a pair
constexpr int kTileN = 256;              // most j of a tile
constexpr int kDeepBytes = 128;          // depth of one ring slot: one swizzle row
constexpr int kDeep = kDeepBytes / 2;    // in bf16 values
constexpr int kPlanPairs = 74;           // the plan is the same on every device: it counts with the pairs of 148 SMs
constexpr int kMostSplits = 32;
constexpr int kMostParts = 4 * kPlanPairs;       // tiles of all splits together, where k is split

// The pass over the output's gradient: tokens that a thread has in flight, and CTAs an SM.  More CTAs of one token each (8192 x 2816 with silu and
// 8-bit pre 52 us with a small product behind it, two tokens and four CTAs 56).
constexpr int kGradPreAhead = 1, kGradPreCtas = 6;

struct LinearPlan {
    int n, splits, per_split;
};

inline int64_t deep_blocks(int64_t k, int deep) { return (k + deep - 1) / deep; }

// n and the number of splits with the least estimated cycles: waves of tiles, a block of k taking 2n cycles on the tensor cores (at least
// what its loads take), a fixed part for filling and emptying a tile, and the parts' way through L2 where k is split.  The last three
// numbers are fitted to 40 products of 8 to 4096 by 256 to 8192 with k of 1024 to 8192, every n and up to 16 splits each: the chosen pair
// takes 1.3 % more than the best one on average and 9 % at most (300 x 7168 to 4096: 23 us, 28 without a split).
inline LinearPlan linear_plan(int64_t I, int64_t J, int64_t blocks)
{
    static const int kSplits[] = {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32};
    LinearPlan best = {32, 1, static_cast<int>(blocks)};
    double least = 1e300;
    const int64_t m_tiles = (I + kTileM - 1) / kTileM;
    for (int n = 32; n <= kTileN; n += 32) {
        if (n > 32 && n - 32 >= J) break;
        const int64_t tiles = m_tiles * ((J + n - 1) / n);
        const double block = 2.0 * n + 64.0 > 400.0 ? 2.0 * n + 64.0 : 400.0;
        for (int s : kSplits) {
            if (s > 1 && (s > blocks || tiles * s > kMostParts || tiles >= 2 * kPlanPairs)) break;
            const int64_t per = (blocks + s - 1) / s, waves = (tiles * s + kPlanPairs - 1) / kPlanPairs;
            if (per * (s - 1) >= blocks) continue;                 // a split without blocks
            double cycles = static_cast<double>(waves) * (per * block + 800.0) + 2500.0;
            if (s > 1) cycles += 3500.0 + s * (450.0 + static_cast<double>(I) * J * 8.0 / 2000.0);
            if (cycles < least) {
                least = cycles;
                best = {n, s, static_cast<int>(per)};
            }
        }
    }
    return best;
}

// At least what the plan's parts take, for J of j and k of `blocks` blocks or fewer: k is split where there are fewer than 2 kPlanPairs tiles,
// into no more parts than it has blocks.
inline size_t part_bytes(int64_t I, int64_t J, int64_t blocks)
{
    const int64_t most_j = (2 * kPlanPairs - 1) / ((I + kTileM - 1) / kTileM) * kTileN, splits = blocks < kMostSplits ? blocks : kMostSplits;
    if (splits < 2) return 0;
    if (J > most_j) J = most_j;
    const int64_t by_splits = splits * I * J, by_tiles = static_cast<int64_t>(kMostParts) * kTileM * kTileN;
    return static_cast<size_t>(by_splits < by_tiles ? by_splits : by_tiles) * sizeof(float);
}

// Slices of the tokens in the pass over the output's gradient: a CTA for every place on an SM, of as equal a number of steps as can be.
inline int bias_parts(int64_t T, int N)
{
    const int64_t groups = (N + 127) / 128, steps = (T + 16 * kGradPreAhead - 1) / (16 * kGradPreAhead);
    int64_t parts = (kGradPreCtas * 2 * kPlanPairs + groups - 1) / groups;
    if (parts > steps) parts = steps;
    if (parts < 1) parts = 1;
    const int64_t each = (steps + parts - 1) / parts;
    return static_cast<int>((steps + each - 1) / each);
}

// The sums of the bias's gradient, for T tokens or fewer.
inline size_t bias_bytes(int64_t T, int32_t N)
{
    const int64_t groups = (N + 127) / 128, steps = (T + 16 * kGradPreAhead - 1) / (16 * kGradPreAhead);
    const int64_t most = (kGradPreCtas * 2 * kPlanPairs + groups - 1) / groups;
    return static_cast<size_t>(steps < most ? steps : most) * N * sizeof(float);
}

// For the forward product (k over K, at most as many blocks as bf16 has), dx (over N) and dW (over T), and the bias's sums.  Never less than for
// fewer tokens.
inline size_t linear_workspace(int64_t T, int32_t K, int32_t N)
{
    if (T == 0) return 256;
    size_t most = bias_bytes(T, N);
    const size_t all[3] = {part_bytes(N, T, deep_blocks(K, kDeep)), part_bytes(K, T, deep_blocks(N, kDeep)), part_bytes(K, N, deep_blocks(T, kDeep))};
    for (size_t b : all) most = b > most ? b : most;
    return ((most > 0 ? most : 1) + 255) / 256 * 256;
}

}  // namespace cobalt
