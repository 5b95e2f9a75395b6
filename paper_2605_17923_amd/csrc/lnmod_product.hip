// lnmod_product.hip -- which kernel computes a product of 8-bit codes, and its launch.
#include <cmath>

#include "lnmod_product_kernels.hpp"

namespace lnmod {
namespace {

constexpr uint32_t kRowOfBlocks = uint32_t{1} << 21;   // a dimension of a grid has fewer than 2^32 threads

// What a launch takes, in microseconds, by counting: `start`, and for each round of blocks over the 256 CUs `tile`, and `step`
// for each of the steps that a block's teams take in turn, `more` for each further block that shares a CU's round.  The
// numbers are least squares to 173 random products of int8 codes and 87 of e4m3 codes to float32 (M 1 to 12 000, N 16 to
// 16 384, K 136 to 14 400, half of the N no multiples of 8) with every one of these kernels.  The kernel that this picks takes
// 1.026 of the fastest one's time in the mean and 1.05 in nine of ten (float32 from e4m3 1.003, 1.00).  The kernel for few rows
// was measured by itself, on 400 problems of up to 16 rows against the first three of the others: 1.04 and 1.13 (with blocks of
// sixteen waves 1.08, 1.23; of four waves with four steps under way 1.07, 1.21).  One kernel
// for all int8 problems would take in the mean 1.5 (32 x 64), 1.7 (64 x 64), 2.1 (32 x 32), 2.6 (128 x 128) or 4.5 (256 x 256)
// times the fastest one's time, each of them 3 to 14 times at its worst.
struct Cost {
    float step, more, tile, start;
};
struct Variant {
    int bm, bn, groups, per_cu;        // per_cu: blocks that LDS or registers let share a CU
    Cost cost[2];                      // one instruction for a product's eight bits, or four through half precision
};
constexpr Variant kVariants[] = {
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

double microseconds(const Variant& v, const Cost& c, int64_t M, int64_t N, int64_t K) {
    const double tiles = static_cast<double>((M + v.bm - 1) / v.bm) * static_cast<double>((N + v.bn - 1) / v.bn);
    const int64_t steps = ((K + kBlockK - 1) / kBlockK + v.groups - 1) / v.groups;
    const double all = kNumCU * v.per_cu, rounds = std::floor(tiles / all), left = tiles - rounds * all;
    const auto round = [&](double share) { return share == 0.0 ? 0.0 : (c.step + (share - 1.0) * c.more) * steps + c.tile; };
    return c.start + rounds * round(v.per_cu) + round(std::ceil(left / kNumCU));
}

int pick(int64_t M, int64_t N, int64_t K, bool halves) {
    int best = -1;
    double least = 0.0;
    for (int i = 0; i <= kLarge; ++i) {
        const Variant& v = kVariants[i];
        if ((i == kFew && M > 16) || (i == kLarge && (K <= kBlockK || halves))) continue;
        if ((M + v.bm - 1) / v.bm >= (int64_t{1} << 31) / ((N + v.bn - 1) / v.bn)) continue;      // tiles are counted in 31 bits
        const double t = microseconds(v, v.cost[halves], M, N, K);
        if (best < 0 || t < least) {
            best = i;
            least = t;
        }
    }
    return best;
}

template <typename C, typename Tag, int BM, int BN, int WM, int WN, int STAGES, int GROUPS>
void tiles(ProductArgs a, hipStream_t st) {
    deal_tiles(a, BM, BN);
    const uint32_t x = a.tiles < kRowOfBlocks ? a.tiles : kRowOfBlocks;
    hipLaunchKernelGGL((product_tile_kernel<C, Tag, BM, BN, WM, WN, STAGES, GROUPS>), dim3(x, (a.tiles + x - 1) / x), dim3(GROUPS * WM * WN * kWave), 0, st, a);
}

template <typename C, typename Tag>
hipError_t go(ProductArgs a, hipStream_t st) {
    constexpr bool kHalves = std::is_same<C, e4m3_code>::value && std::is_same<Tag, f32_io>::value;
    switch (pick(a.M, a.N, a.K, kHalves)) {
        case kFew: {
            const uint32_t blocks = static_cast<uint32_t>((a.N + 15) / 16), x = blocks < kRowOfBlocks ? blocks : kRowOfBlocks;
            hipLaunchKernelGGL((product_few_kernel<C, Tag, 1, 1, 2, 8>), dim3(x, (blocks + x - 1) / x), dim3(8 * kWave), 0, st, a);
            break;
        }
        case 1: tiles<C, Tag, 32, 32, 2, 1, 4, 4>(a, st); break;
        case 2: tiles<C, Tag, 32, 64, 2, 2, 3, 2>(a, st); break;
        case 3: tiles<C, Tag, 64, 64, 2, 2, 3, 2>(a, st); break;
        case 4: tiles<C, Tag, 96, 64, 2, 2, 3, 2>(a, st); break;
        case 5: tiles<C, Tag, 128, 64, 2, 2, 3, 2>(a, st); break;
        case 6: tiles<C, Tag, 128, 128, 4, 2, 4, 1>(a, st); break;
        case 7: tiles<C, Tag, 128, 128, 2, 2, 2, 1>(a, st); break;
        case 8: tiles<C, Tag, 128, 256, 2, 4, 3, 1>(a, st); break;
        case kLarge:
            if constexpr (!kHalves) {
                deal_tiles(a, 256, 256);
                hipLaunchKernelGGL((product_large_kernel<C, Tag>), dim3(a.tiles < kNumCU ? a.tiles : kNumCU), dim3(8 * kWave), 0, st, a);
            }
            break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace

// Outputs beyond 64 MB go past the caches (8192 x 13 824 bf16 549 -> 463 us, 8192 x 8192 478 -> 418, 4096 x 4096 58.1 and 58.9)
// where every row of them is whole lines.
hipError_t launch_product(int dtype, int code, ProductArgs a, hipStream_t st) {
    const int64_t row = a.N * (dtype == 0 ? 2 : 4);
    a.keep = row % 128 != 0 || a.M * row <= (int64_t{64} << 20);
    a.wide = reinterpret_cast<uintptr_t>(a.bias) % 4 == 0;
    if (code == 0) return dtype == 0 ? go<int8_code, bf16_io>(a, st) : go<int8_code, f32_io>(a, st);
    return dtype == 0 ? go<e4m3_code, bf16_io>(a, st) : go<e4m3_code, f32_io>(a, st);
}

}  // namespace lnmod
