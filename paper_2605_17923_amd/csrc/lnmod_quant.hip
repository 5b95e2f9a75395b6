// lnmod_quant.hip -- instantiation and launch of the 8-bit checkpoint of a tensor and the way back.
#include "lnmod_launch.hpp"
#include "lnmod_quant_kernels.hpp"

namespace lnmod {
namespace {

constexpr int kPieces = 4;           // pieces per wave and step
constexpr int kBlocksPerCu = 4;

template <bool BACK>
hipError_t launch(int dtype, int code, const void* x, void* codes, float* scales, int64_t N, int64_t D, int64_t group,
                  hipStream_t st) {
    QuantArgs a;
    a.x = const_cast<void*>(x);
    a.codes = codes;
    a.scales = scales;
    // group 0 (the way back only): one scale for a row, every unit of which then has the group number 0
    a.lanes_log2 = group == 0 ? 31 : group_lanes_log2(group);
    const int64_t units = D / kUnit;
    a.total = N * units;
    if (group != 0 && D % group == 0) {
        a.units = kWave;
        a.rows = (a.total + kWave - 1) / kWave;
    } else {
        a.units = static_cast<int32_t>(units);
        a.rows = N;
    }
    a.per_row = (a.units + kWave - 1) / kWave;
    a.groups = group == 0 ? 1 : (a.units + (1 << a.lanes_log2) - 1) >> a.lanes_log2;
    const int64_t steps = (a.rows * a.per_row + kPieces - 1) / kPieces;      // of a wave
    int64_t blocks = (steps + kQuantWaves - 1) / kQuantWaves;
    if (blocks > kNumCU * kBlocksPerCu) blocks = kNumCU * kBlocksPerCu;
    const int64_t stride = blocks * kQuantWaves * kPieces;                   // pieces
    a.row_step = stride / a.per_row;
    a.piece_step = static_cast<int32_t>(stride % a.per_row);
    const dim3 grid(static_cast<unsigned>(blocks)), block(kQuantWaves * kWave);
    if (dtype == 0 && code == 0) hipLaunchKernelGGL((quant_kernel<bf16_io, int8_code, kPieces, BACK>), grid, block, 0, st, a);
    else if (dtype == 0) hipLaunchKernelGGL((quant_kernel<bf16_io, e4m3_code, kPieces, BACK>), grid, block, 0, st, a);
    else if (code == 0) hipLaunchKernelGGL((quant_kernel<f32_io, int8_code, kPieces, BACK>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((quant_kernel<f32_io, e4m3_code, kPieces, BACK>), grid, block, 0, st, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize(int dtype, int code, const void* x, int64_t N, int64_t D, int64_t group, void* codes,
                           float* scales, hipStream_t st) {
    return launch<false>(dtype, code, x, codes, scales, N, D, group, st);
}

hipError_t launch_dequantize(int dtype, int code, const void* codes, const float* scales, int64_t N, int64_t D, int64_t group,
                             void* x, hipStream_t st) {
    return launch<true>(dtype, code, x, const_cast<void*>(codes), const_cast<float*>(scales), N, D, group, st);
}

}  // namespace lnmod
