// lnmod_product.hip -- launch of the product of 8-bit codes.
#include "lnmod_product_kernels.hpp"

namespace lnmod {
namespace {

constexpr uint32_t kRowOfBlocks = uint32_t{1} << 22;   // a dimension of a grid has fewer than 2^32 threads

template <typename C, typename Tag>
void go(ProductArgs a, hipStream_t st) {
    a.keep = 0;
    if constexpr (!(std::is_same<C, e4m3_code>::value && std::is_same<Tag, f32_io>::value)) {
        if (a.K > kBlockK && a.M >= 256 && a.N >= 256 && a.M * a.N >= int64_t{64} * 65536) {
            deal_tiles(a, 256, 256);
            hipLaunchKernelGGL((product_large_kernel<C, Tag>), dim3(a.tiles < kNumCU ? a.tiles : kNumCU), dim3(8 * kWave), 0, st, a);
            return;
        }
    }
    deal_tiles(a, 128, 128);
    const uint32_t x = a.tiles < kRowOfBlocks ? a.tiles : kRowOfBlocks;
    hipLaunchKernelGGL((product_tile_kernel<C, Tag, 128, 128, 2, 2>), dim3(x, (a.tiles + x - 1) / x), dim3(4 * kWave), 0, st, a);
}

}  // namespace

hipError_t launch_product(int dtype, int code, const ProductArgs& a, hipStream_t st) {
    if (code == 0) {
        if (dtype == 0) go<int8_code, bf16_io>(a, st);
        else go<int8_code, f32_io>(a, st);
    } else {
        if (dtype == 0) go<e4m3_code, bf16_io>(a, st);
        else go<e4m3_code, f32_io>(a, st);
    }
    return hipGetLastError();
}

}  // namespace lnmod
