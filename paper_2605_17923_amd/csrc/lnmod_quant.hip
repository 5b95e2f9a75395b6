// lnmod_quant.hip -- instantiation and launch of the 8-bit checkpoint of a tensor and the way back.
#include "lnmod_launch.hpp"
#include "lnmod_quant_kernels.hpp"

namespace lnmod {
namespace {

// Pieces a wave takes per step, and blocks per CU that the grid has at most (many more than are resident: with four,
// 75 600 x 5120 bf16 took 211 us there and 217 back, with 64 it takes 187 and 194; 10 000 x 5120 30.8 and 31.4, with 32 of two
// pieces 26.7 and 27.4).  Small launches take one piece a wave, so that every CU has a part (200 x 5120 3.9 -> 2.7 us, 1025 x 1432
// 4.3 -> 3.3); fp32 units are 32 bytes of a lane and always take one (20 000 x 5120 97 and 134 -> 88 and 95).
struct QuantShape {
    int pieces, per_cu;
};
QuantShape quant_shape(int64_t bytes, int dtype) {
    if (dtype != 0) return {1, 1 << 20};
    if (bytes <= 16000000) return {1, 16};
    return bytes <= 300000000 ? QuantShape{2, 32} : QuantShape{4, 64};
}

template <bool BACK>
hipError_t launch(int dtype, int code, const void* x, void* codes, float* scales, int64_t N, int64_t D, int64_t group,
                  hipStream_t st) {
    QuantArgs a;
    a.x = const_cast<void*>(x);
    a.codes = codes;
    a.scales = scales;
    // group 0 (the way back only): one scale for a row, every unit of which then has the group number 0
    a.lanes_log2 = group == 0 ? 31 : group_lanes_log2(group);
    a.keep = keep_codes(N, D, 0, 4000000);
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
    const QuantShape sh = quant_shape(N * D * (dtype == 0 ? 2 : 4), dtype);
    const int64_t steps = (a.rows * a.per_row + sh.pieces - 1) / sh.pieces;  // of a wave
    int64_t blocks = (steps + kQuantWaves - 1) / kQuantWaves;
    if (blocks > int64_t(kNumCU) * sh.per_cu) blocks = int64_t(kNumCU) * sh.per_cu;
    const int64_t stride = blocks * kQuantWaves * sh.pieces;                 // pieces
    a.row_step = stride / a.per_row;
    a.piece_step = static_cast<int32_t>(stride % a.per_row);
    const dim3 grid(static_cast<unsigned>(blocks)), block(kQuantWaves * kWave);
    const auto run = [&](auto io, auto cd, auto pieces) {
        hipLaunchKernelGGL((quant_kernel<decltype(io), decltype(cd), pieces, BACK>), grid, block, 0, st, a);
    };
    const auto coded = [&](auto io, auto pieces) {
        if (code == 0) run(io, int8_code{}, pieces);
        else run(io, e4m3_code{}, pieces);
    };
    using std::integral_constant;
    if (dtype != 0) coded(f32_io{}, integral_constant<int, 1>{});
    else if (sh.pieces == 1) coded(bf16_io{}, integral_constant<int, 1>{});
    else if (sh.pieces == 2) coded(bf16_io{}, integral_constant<int, 2>{});
    else coded(bf16_io{}, integral_constant<int, 4>{});
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
