// lnmod_product.hip -- instantiation and launch of the product of 8-bit codes (lnmod_product_plan.hpp says by which kernel).
#include "lnmod_product_kernels.hpp"

namespace lnmod {
namespace {

constexpr uint32_t kRowOfBlocks = uint32_t{1} << 21;   // a dimension of a grid has fewer than 2^32 threads

template <typename C, typename Tag, int BM, int BN, int WM, int WN, int STAGES, int GROUPS>
void tiles(ProductArgs a, hipStream_t st) {
    deal_tiles(a, BM, BN);
    const uint32_t x = a.tiles < kRowOfBlocks ? a.tiles : kRowOfBlocks;
    hipLaunchKernelGGL((product_tile_kernel<C, Tag, BM, BN, WM, WN, STAGES, GROUPS>), dim3(x, (a.tiles + x - 1) / x), dim3(GROUPS * WM * WN * kWave), 0, st, a);
}

template <typename C, typename Tag>
hipError_t go(ProductArgs a, hipStream_t st) {
    constexpr bool kHalves = std::is_same<C, e4m3_code>::value && std::is_same<Tag, f32_io>::value;
    switch (pick_product(a.M, a.N, a.K, kHalves)) {
        case kFew: {
            const uint32_t blocks = static_cast<uint32_t>((a.N + kFewOutputs - 1) / kFewOutputs), x = blocks < kRowOfBlocks ? blocks : kRowOfBlocks;
            hipLaunchKernelGGL((product_few_kernel<C, Tag>), dim3(x, (blocks + x - 1) / x), dim3(kFewWaves * kWave), 0, st, a);
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

hipError_t launch_product(int dtype, int code, ProductArgs a, hipStream_t st) {
    a.keep = keeps_products(a.M, a.N, dtype == 0 ? 2 : 4);
    a.wide = reinterpret_cast<uintptr_t>(a.bias) % 4 == 0;
    if (code == 0) return dtype == 0 ? go<int8_code, bf16_io>(a, st) : go<int8_code, f32_io>(a, st);
    return dtype == 0 ? go<e4m3_code, bf16_io>(a, st) : go<e4m3_code, f32_io>(a, st);
}

}  // namespace lnmod
