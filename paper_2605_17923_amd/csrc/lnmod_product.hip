// lnmod_product.hip -- launch of the product of 8-bit codes.
#include "lnmod_product_kernels.hpp"

namespace lnmod {
namespace {

constexpr int64_t kRowOfBlocks = int64_t{1} << 22;   // a dimension of a grid has fewer than 2^32 threads

template <typename C, typename Tag>
void go(ProductArgs a, hipStream_t st) {
    if constexpr (!(std::is_same<C, e4m3_code>::value && std::is_same<Tag, f32_io>::value)) {
        if (a.M >= 256 && a.N >= 256 && a.M * a.N >= int64_t{64} * 65536) {
            a.tiles_m = static_cast<int32_t>((a.M + 255) / 256);
            a.tiles = static_cast<int64_t>(a.tiles_m) * ((a.N + 255) / 256);
            const int64_t blocks = a.tiles < kNumCU ? a.tiles : kNumCU;
            hipLaunchKernelGGL((product_large_kernel<C, Tag>), dim3(static_cast<unsigned>(blocks)), dim3(512), 0, st, a);
            return;
        }
    }
    constexpr int BM = 128, BN = 128;
    a.tiles_m = static_cast<int32_t>((a.M + BM - 1) / BM);
    a.tiles = static_cast<int64_t>(a.tiles_m) * ((a.N + BN - 1) / BN);
    const int64_t x = a.tiles < kRowOfBlocks ? a.tiles : kRowOfBlocks;
    const dim3 grid(static_cast<unsigned>(x), static_cast<unsigned>((a.tiles + x - 1) / x));
    hipLaunchKernelGGL((product_tile_kernel<C, Tag, BM, BN, 2, 2>), grid, dim3(256), 0, st, a);
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
