// lnmod_rmsq.hip -- instantiation and launch of the root-mean-square norm with the residual's addition and an output in
// 8 bits, and of its backward.
#include "lnmod_launch.hpp"
#include "lnmod_rmsq_kernels.hpp"

namespace lnmod {
namespace {

// Two units per lane, as many waves as the row then needs.
Shape rmsq_shape(int units, int dtype) {
    Shape sh{1, 1, dtype == 0 ? 2 : 1, 8};
    if (units > kWave) {
        sh.VPL = 2;
        sh.K = (units + 2 * kWave - 1) / (2 * kWave);
        if (sh.K == 7) sh.K = 8;
        sh.per_cu = sh.K <= 1 ? 8 : sh.K == 2 ? 4 : sh.K <= 4 ? 2 : 1;
    }
    return sh;
}

Shape rmsq_fwd_shape(int units, int dtype, int64_t) { return rmsq_shape(units, dtype); }
Shape rmsq_bwd_shape(int units, int dtype) { return rmsq_shape(units, dtype); }

int64_t blocks_for(int64_t N, const Shape& sh) { return grid_blocks(N, static_cast<int64_t>(kNumCU) * sh.per_cu, sh.R); }

// f(VPL, K, R) as constants; false for a shape that is not compiled
template <typename F>
bool for_shape(const Shape& sh, F&& f) {
    using std::integral_constant;
    const auto rows = [&](auto vpl, auto k) {
        if (sh.R == 1) f(vpl, k, integral_constant<int, 1>{});
        else f(vpl, k, integral_constant<int, 2>{});
        return true;
    };
    switch (sh.VPL * 100 + sh.K) {
        case 101: return rows(integral_constant<int, 1>{}, integral_constant<int, 1>{});
        case 201: return rows(integral_constant<int, 2>{}, integral_constant<int, 1>{});
        case 202: return rows(integral_constant<int, 2>{}, integral_constant<int, 2>{});
        case 203: return rows(integral_constant<int, 2>{}, integral_constant<int, 3>{});
        case 204: return rows(integral_constant<int, 2>{}, integral_constant<int, 4>{});
        case 205: return rows(integral_constant<int, 2>{}, integral_constant<int, 5>{});
        case 206: return rows(integral_constant<int, 2>{}, integral_constant<int, 6>{});
        case 208: return rows(integral_constant<int, 2>{}, integral_constant<int, 8>{});
        default: return false;
    }
}

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
    a.eps = eps;
    a.inv_D = 1.0f / static_cast<float>(D);
    const Shape sh = pick_shape(force, rmsq_fwd_shape(a.nchunks, dtype, N));
    if (!covers(sh, a.nchunks)) return hipErrorInvalidConfiguration;
    a.nb = static_cast<int32_t>(blocks_for(N, sh));
    const dim3 grid(static_cast<unsigned>(a.nb)), block(sh.K * kWave);
    const auto run = [&](auto io, auto cd) {
        return for_shape(sh, [&](auto vpl, auto k, auto rows) {
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
        });
    };
    bool ok;
    if (dtype == 0) ok = code == 0 ? run(bf16_io{}, int8_code{}) : run(bf16_io{}, e4m3_code{});
    else ok = code == 0 ? run(f32_io{}, int8_code{}) : run(f32_io{}, e4m3_code{});
    return ok ? hipGetLastError() : hipErrorInvalidConfiguration;
}

int64_t rmsq_bwd_blocks(int64_t N, int64_t D, int dtype) {
    return N <= 0 ? 0 : blocks_for(N, rmsq_bwd_shape(static_cast<int>(D / kUnit), dtype));
}

hipError_t launch_rmsq_bwd(int dtype, const void* dy, const void* dh, const void* h, const void* w, int64_t N, int64_t D,
                           const float* rstd, void* dx, void* dw, bool io_grads, float* ws, hipStream_t st, const Shape* force) {
    RmsqBwdArgs a{};
    a.dy = dy;
    a.dh = dh;
    a.h = h;
    a.w = w;
    a.rstd = rstd;
    a.dx = dx;
    a.ws = ws;
    a.N = N;
    a.D = static_cast<int32_t>(D);
    a.nchunks = static_cast<int32_t>(D / kUnit);
    a.inv_D = 1.0f / static_cast<float>(D);
    const Shape sh = pick_shape(force, rmsq_bwd_shape(a.nchunks, dtype));
    if (!covers(sh, a.nchunks)) return hipErrorInvalidConfiguration;
    a.nb = static_cast<int32_t>(blocks_for(N, sh));
    const dim3 grid(static_cast<unsigned>(a.nb)), block(sh.K * kWave);
    const auto run = [&](auto io) {
        return for_shape(sh, [&](auto vpl, auto k, auto rows) {
            using Tag = decltype(io);
            if (dh) hipLaunchKernelGGL((rmsq_bwd_kernel<Tag, vpl, k, rows, true>), grid, block, 0, st, a);
            else hipLaunchKernelGGL((rmsq_bwd_kernel<Tag, vpl, k, rows, false>), grid, block, 0, st, a);
        });
    };
    if (!(dtype == 0 ? run(bf16_io{}) : run(f32_io{}))) return hipErrorInvalidConfiguration;
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
