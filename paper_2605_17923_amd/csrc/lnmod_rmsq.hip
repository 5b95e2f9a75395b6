// lnmod_rmsq.hip -- instantiation and launch of the root-mean-square norm with the residual's addition and an output in
// 8 bits, and of its backward.
#include <algorithm>

#include "lnmod_code_shapes.hpp"
#include "lnmod_rmsq_kernels.hpp"

namespace lnmod {
namespace {

int64_t fwd_blocks_for(int64_t N, const Shape& sh) {
    const int groups = fwd_row_groups(N, sh);
    return grid_blocks(N, static_cast<int64_t>(kNumCU) * sh.per_cu / groups, sh.R * groups);
}
// see groups_fit in lnmod_ckpt.hip
template <typename Tag>
constexpr bool groups_fit(const ShapeTable& t, bool dh) {
    for (const Shape& s : t)
        if (s.K == 1 && s.per_cu > groups_most(1, rmsq_bwd_waves(s.VPL, Unit<Tag>::NV, s.R, dh))) return false;
    return true;
}
static_assert(groups_fit<bf16_io>(kRmsBwd50, true) && groups_fit<bf16_io>(kRmsBwd50, false) && groups_fit<bf16_io>(kRmsBwdLong, true) &&
              groups_fit<bf16_io>(kRmsBwdLongAlone, false) && groups_fit<f32_io>(kRmsBwd50x32, true) &&
              groups_fit<f32_io>(kRmsBwd50x32, false) && groups_fit<f32_io>(kRmsBwd32, true) && groups_fit<f32_io>(kRmsBwd32, false),
              "more waves than the kernel's launch bounds");
int64_t bwd_blocks_for(int64_t N, const Shape& sh) { return grid_blocks(N, group_blocks_most(sh), sh.R * row_groups(N, sh)); }

}  // namespace

hipError_t launch_rmsq_fwd(int dtype, int code, const void* x, const void* r, const void* w, int64_t N, int64_t D, float eps,
                           int64_t group, void* h, void* out, float* scales, float* rstd, bool values, hipStream_t st,
                           const Shape* force) {
    RmsqFwdArgs a{};
    a.x = x;
    a.r = r;
    a.w = w;
    a.h = h;
    a.out = out;
    a.scales = scales;
    a.rstd = rstd;
    a.N = N;
    a.D = static_cast<int32_t>(D);
    a.nchunks = static_cast<int32_t>(D / kUnit);
    a.lanes_log2 = group == 0 ? 0 : group_lanes_log2(group);
    a.groups = group == 0 ? 1 : static_cast<int32_t>((D + group - 1) / group);
    a.keep = keep_codes(N, D, 0, r ? 70000000 : 4000000);
    a.eps = eps;
    a.inv_D = 1.0f / static_cast<float>(D);
    const Shape sh = pick_shape(force, rms_fwd_shape(N, a.nchunks, dtype));
    if (!covers(sh, a.nchunks)) return hipErrorInvalidConfiguration;
    a.nb = static_cast<int32_t>(fwd_blocks_for(N, sh));
    const dim3 grid(static_cast<unsigned>(a.nb)), block(sh.K * fwd_row_groups(N, sh) * kWave);
    const auto run = [&](auto io, auto cd) {
        const auto shaped = [&](auto vpl, auto k, auto rows) {
            const auto go = [&](auto res, auto row, auto val) {
                hipLaunchKernelGGL((rmsq_fwd_kernel<decltype(io), decltype(cd), vpl, k, rows, res, row, val>), grid, block, 0, st, a);
            };
            const auto with = [&](auto res, auto row) {
                if (values) go(res, row, std::true_type{});
                else go(res, row, std::false_type{});
            };
            const auto res = [&](auto has) {
                if (group == 0) with(has, std::true_type{});
                else with(has, std::false_type{});
            };
            if (r) res(std::true_type{});
            else res(std::false_type{});
        };
        if constexpr (std::is_same<decltype(io), bf16_io>::value) return ShapesOf<kSplit, kRmsFwd200, kRmsFwdLong>::call(sh, shaped);
        else return ShapesOf<kSplit, kRmsFwd32>::call(sh, shaped);
    };
    bool ok;
    if (dtype == 0) ok = code == 0 ? run(bf16_io{}, int8_code{}) : run(bf16_io{}, e4m3_code{});
    else ok = code == 0 ? run(f32_io{}, int8_code{}) : run(f32_io{}, e4m3_code{});
    return ok ? hipGetLastError() : hipErrorInvalidConfiguration;
}

int64_t rmsq_bwd_most_slots(int64_t N, int64_t D, int dtype) {
    if (N <= 0) return 0;
    const int units = static_cast<int>(D / kUnit);
    return std::max(most_slots(N, rms_bwd_shape(N, units, dtype, false)), most_slots(N, rms_bwd_shape(N, units, dtype, true)));
}

hipError_t launch_rmsq_bwd(int dtype, const void* dy, const void* dh, const void* h, const void* w, int64_t N, int64_t D,
                           const float* rstd, void* dx, void* dr, void* dw, bool io_grads, float* ws, hipStream_t st, const Shape* force) {
    RmsqBwdArgs a{};
    a.dy = dy;
    a.dh = dh;
    a.h = h;
    a.w = w;
    a.rstd = rstd;
    a.dx = dx;
    a.dr = dr;
    a.ws = ws;
    a.N = N;
    a.D = static_cast<int32_t>(D);
    a.nchunks = static_cast<int32_t>(D / kUnit);
    a.inv_D = 1.0f / static_cast<float>(D);
    const Shape sh = pick_shape(force, rms_bwd_shape(N, a.nchunks, dtype, dh != nullptr));
    if (!covers(sh, a.nchunks)) return hipErrorInvalidConfiguration;
    a.nb = static_cast<int32_t>(bwd_blocks_for(N, sh));
    const int groups = row_groups(N, sh);
    bool fits = true;
    const dim3 grid(static_cast<unsigned>(a.nb)), block(sh.K * groups * kWave);
    const auto run = [&](auto io) {
        const auto go = [&](auto vpl, auto k, auto rows) {
            using Tag = decltype(io);
            const auto add = [&](auto has) {
                constexpr int waves = rmsq_bwd_waves(vpl, Unit<Tag>::NV, rows, has);
                const size_t lds = group_lds(groups, units_at_once(vpl, waves), 1);
                fits = groups <= groups_most(k, waves);
                if (fits) hipLaunchKernelGGL((rmsq_bwd_kernel<Tag, vpl, k, rows, has>), grid, block, lds, st, a);
            };
            if (dh) add(std::true_type{});
            else add(std::false_type{});
        };
        if constexpr (std::is_same<decltype(io), bf16_io>::value) return ShapesOf<kRmsBwd50, kRmsBwdLong, kRmsBwdLongAlone>::call(sh, go);
        else return ShapesOf<kRmsBwd50x32, kRmsBwd32>::call(sh, go);
    };
    if (!(dtype == 0 ? run(bf16_io{}) : run(f32_io{})) || !fits) return hipErrorInvalidConfiguration;
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;

    ReduceArgs r{};
    r.ws = ws;
    r.out[0] = dw;
    r.out_bf16 = io_grads && dtype == 0;
    r.seg = Segments{nullptr, N, 1};
    r.T = N;
    r.rows_per_cluster = N;
    r.nb = a.nb;
    r.D = a.D;
    r.nsum = 1;
    return launch_reduce(r, 1, st);
}

}  // namespace lnmod
