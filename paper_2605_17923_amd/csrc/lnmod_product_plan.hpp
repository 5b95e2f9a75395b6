// lnmod_product_plan.hpp -- which kernel computes a product of 8-bit codes, and where its outputs go.  Host code.
#pragma once
#include <cmath>

#include "lnmod_launch.hpp"

namespace lnmod {

constexpr int kBlockK = 128;                 // features of a step: one cache line of a row

// What a launch takes, in microseconds, by counting: `start`, and for each round of blocks over the 256 CUs `tile`, and `step`
// for each of the steps that a block's teams take in turn, `more` for each further block that shares a CU's round.  The
// numbers are least squares to 173 random products of int8 codes and 87 of e4m3 codes to float32 (M 1 to 12 000, N 16 to
// 16 384, K 136 to 14 400, half of the N no multiples of 8) with every one of these kernels.  The kernel that this picks takes
// 1.026 of the fastest one's time in the mean and 1.05 in nine of ten (float32 from e4m3 1.003, 1.00).  The kernel for few rows
// was measured by itself, on 400 problems of up to 16 rows against the first three of the others: 1.04 and 1.13 (with blocks of
// sixteen waves 1.08, 1.23; of four waves with four steps under way 1.07, 1.21).  One kernel
// for all int8 problems would take in the mean 1.5 (32 x 64), 1.7 (64 x 64), 2.1 (32 x 32), 2.6 (128 x 128) or 4.5 (256 x 256)
// times the fastest one's time, each of them 3 to 14 times at its worst.
//
// int8 codes to float32 and e4m3 codes to bf16 go by the first column too, which was fitted to int8 codes to bf16.  The operands were
// eight sets in turn, so weights below about 30 MB came from the last-level cache and larger ones from HBM; no term counts bytes.
struct ProductCost {
    float step, more, tile, start;
};
struct ProductKernel {
    int bm, bn, groups, per_cu;        // per_cu: blocks that LDS or registers let share a CU
    ProductCost cost[2];               // one instruction for a product's eight bits, or four through half precision
};
constexpr ProductKernel kProducts[] = {
    {16, 16, 8, 2, {{0.470f, 0.939f, 0.0f, 2.14f}, {0.499f, 0.853f, 0.0f, 2.14f}}},      // few rows
    {32, 32, 4, 1, {{0.452f, 0.0f, 1.77f, 1.43f}, {0.614f, 0.0f, 1.76f, 1.31f}}},
    {32, 64, 2, 2, {{0.328f, 0.338f, 1.51f, 2.05f}, {0.488f, 0.324f, 1.73f, 1.94f}}},
    {64, 64, 2, 1, {{0.473f, 0.0f, 2.32f, 1.47f}, {0.647f, 0.0f, 3.03f, 1.09f}}},
    {96, 64, 2, 1, {{0.592f, 0.0f, 2.88f, 1.09f}, {0.837f, 0.0f, 3.83f, 0.31f}}},
    {128, 64, 2, 1, {{0.726f, 0.0f, 3.34f, 0.87f}, {1.035f, 0.0f, 4.28f, 0.0f}}},
    {128, 128, 1, 1, {{0.552f, 0.0f, 3.98f, 0.0f}, {0.930f, 0.0f, 4.09f, 0.0f}}},        // eight waves, four steps in LDS
    {128, 128, 1, 2, {{0.690f, 0.463f, 4.05f, 0.55f}, {0.962f, 0.582f, 4.73f, 0.0f}}},   // four waves, two steps
    {128, 256, 1, 1, {{0.859f, 0.0f, 4.85f, 0.0f}, {1.480f, 0.0f, 4.55f, 0.0f}}},
    {256, 256, 1, 1, {{1.189f, 0.0f, 9.51f, 0.0f}, {1e9f, 0.0f, 0.0f, 0.0f}}}};          // large
constexpr int kFew = 0, kLarge = 9;

inline double product_microseconds(const ProductKernel& v, const ProductCost& c, int64_t M, int64_t N, int64_t K) {
    const double tiles = static_cast<double>((M + v.bm - 1) / v.bm) * static_cast<double>((N + v.bn - 1) / v.bn);
    const int64_t steps = ((K + kBlockK - 1) / kBlockK + v.groups - 1) / v.groups;
    const double all = kNumCU * v.per_cu, rounds = std::floor(tiles / all), left = tiles - rounds * all;
    const auto round = [&](double share) { return share == 0.0 ? 0.0 : (c.step + (share - 1.0) * c.more) * steps + c.tile; };
    return c.start + rounds * round(v.per_cu) + round(std::ceil(left / kNumCU));
}

// The kernel for a product, an index of kProducts.  halves: e4m3 codes to float32.
inline int pick_product(int64_t M, int64_t N, int64_t K, bool halves) {
    int best = -1;
    double least = 0.0;
    for (int i = 0; i <= kLarge; ++i) {
        const ProductKernel& v = kProducts[i];
        if ((i == kFew && M > 16) || (i == kLarge && (K <= kBlockK || halves))) continue;
        if ((M + v.bm - 1) / v.bm >= (int64_t{1} << 31) / ((N + v.bn - 1) / v.bn)) continue;      // tiles are counted in 31 bits
        const double t = product_microseconds(v, v.cost[halves], M, N, K);
        if (best < 0 || t < least) {
            best = i;
            least = t;
        }
    }
    return best;
}

// Outputs beyond 64 MB go past the caches (8192 x 13 824 bf16 549 -> 463 us, 8192 x 8192 478 -> 418, 4096 x 4096 58.1 and 58.9)
// where every row of them is whole lines.
inline bool keeps_products(int64_t M, int64_t N, int64_t bytes) {
    const int64_t row = N * bytes;
    return row % 128 != 0 || M * row <= (int64_t{64} << 20);
}

}  // namespace lnmod
