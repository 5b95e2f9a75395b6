// lnmod_quant.hip -- instantiation and launch of the 8-bit checkpoint of a tensor and the way back.
#include "lnmod_code_shapes.hpp"
#include "lnmod_launch.hpp"
#include "lnmod_quant_kernels.hpp"

namespace lnmod {
namespace {

template <bool BACK>
hipError_t launch(int dtype, int code, const void* x, void* codes, float* scales, int64_t N, int64_t D, int64_t group,
                  hipStream_t st) {
    QuantArgs a{};
    a.x = const_cast<void*>(x);
    a.codes = codes;
    a.scales = scales;
    // group 0 (the way back only): one scale for a row, every unit of which then has the group number 0
    a.lanes_log2 = group == 0 ? 31 : group_lanes_log2(group);
    a.keep = keep_codes(N, D, 0, 4000000);
    const bool pad = group == 0 || D % group != 0;
    a.units = static_cast<int32_t>(D / kUnit);
    a.total = N * a.units;
    a.groups = group == 0 ? 1 : (a.units + (1 << a.lanes_log2) - 1) >> a.lanes_log2;
    a.slots = pad && !BACK ? a.groups << a.lanes_log2 : a.units;
    const int64_t pieces = (N * a.slots + kWave - 1) / kWave;
    a.rows = pad ? N : pieces;
    a.rows_in_64 = kWave / a.slots;
    a.left_in_64 = kWave % a.slots;
    a.over_slots = (65536u + static_cast<uint32_t>(a.slots) - 1u) / static_cast<uint32_t>(a.slots);
    const QuantShape sh = quant_shape(N * D * (dtype == 0 ? 2 : 4), dtype);
    const int64_t blocks = quant_blocks(pieces, sh);
    const int64_t stride = blocks * kQuantWaves * sh.pieces;                 // pieces
    a.row_step = pad ? stride * kWave / a.slots : stride;
    a.slot_step = pad ? static_cast<int32_t>(stride * kWave % a.slots) : 0;
    const dim3 grid(static_cast<unsigned>(blocks)), block(kQuantWaves * kWave);
    const auto run = [&](auto io, auto cd, auto v) {
        if (pad) hipLaunchKernelGGL((quant_kernel<decltype(io), decltype(cd), v, BACK, true>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((quant_kernel<decltype(io), decltype(cd), v, BACK, false>), grid, block, 0, st, a);
    };
    const auto coded = [&](auto io, auto v) {
        if (code == 0) run(io, int8_code{}, v);
        else run(io, e4m3_code{}, v);
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
