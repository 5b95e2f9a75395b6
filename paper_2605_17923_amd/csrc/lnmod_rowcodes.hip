// lnmod_rowcodes.hip -- launch of the codes with one scale for a row.
#include "lnmod_rowcodes_kernels.hpp"

namespace lnmod {
namespace {

constexpr int64_t kMostBlocks = int64_t{1} << 20;    // rows beyond that many are taken in turns

template <typename Tag, typename C>
void go(const RowCodesArgs& a, int vpl, unsigned blocks, unsigned threads, hipStream_t st) {
    switch (vpl) {
        case 1: hipLaunchKernelGGL((row_codes_kernel<Tag, C, 1>), dim3(blocks), dim3(threads), 0, st, a); break;
        case 2: hipLaunchKernelGGL((row_codes_kernel<Tag, C, 2>), dim3(blocks), dim3(threads), 0, st, a); break;
        case 4: hipLaunchKernelGGL((row_codes_kernel<Tag, C, 4>), dim3(blocks), dim3(threads), 0, st, a); break;
        default: hipLaunchKernelGGL((long_row_codes_kernel<Tag, C>), dim3(blocks), dim3(threads), 0, st, a); break;
    }
}

}  // namespace

hipError_t launch_row_codes(int dtype, int code, const void* x, int64_t N, int64_t D, void* codes, float* scales, hipStream_t st) {
    RowCodesArgs a{x, codes, scales, N, static_cast<int32_t>(D), static_cast<int32_t>(D / 8), 6, 1, keep_codes(N, D, 0, 128000000)};
    // As many units a lane as a row fills, to have its loads under way at once; blocks of one row each, but of four waves where a
    // wave holds several rows.  400 MB of bf16 and int8, us, with 1, 2 and 4 units a lane (the floor is 105 at 6.0 TB/s, half of it
    // in the 256 MB cache): D 1024 121, 98, -; 1536 127, 114, -; 2048 124, 103, 102; 5120 -, 110, 106; 13 824 -, 124, 105.  fp32,
    // whose loads are two a unit: within 3 % of the best at 26 sizes.
    const int rounds = (a.units + kWave - 1) / kWave;
    int vpl = rounds == 1 ? 1 : rounds <= 3 ? 2 : 4;
    a.waves = (rounds + vpl - 1) / vpl;
    int teams = 1;
    if (a.waves > kRowCodesWaves) {
        vpl = 0;
        a.waves = 1;
    } else if (a.waves == 1) {
        teams = vpl == 1 ? 4 : 1;
        a.lanes_log2 = 0;
        while ((1 << a.lanes_log2) < a.units && a.lanes_log2 < 6) ++a.lanes_log2;
    }
    const int64_t rows = vpl == 0 ? 1 : static_cast<int64_t>(teams) << (6 - a.lanes_log2);
    int64_t blocks = (N + rows - 1) / rows;
    if (blocks > kMostBlocks) blocks = kMostBlocks;
    const unsigned grid = static_cast<unsigned>(blocks), threads = vpl == 0 ? kRowCodesWaves * kWave : teams * a.waves * kWave;
    if (dtype == 0) {
        if (code == 0) go<bf16_io, int8_code>(a, vpl, grid, threads, st);
        else go<bf16_io, e4m3_code>(a, vpl, grid, threads, st);
    } else {
        if (code == 0) go<f32_io, int8_code>(a, vpl, grid, threads, st);
        else go<f32_io, e4m3_code>(a, vpl, grid, threads, st);
    }
    return hipGetLastError();
}

}  // namespace lnmod
