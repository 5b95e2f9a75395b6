// lnmod_ckpt.hip -- instantiation and launch of LayerNorm-Modulate with an 8-bit checkpoint of x: the forward that writes
// it and the backward that reads it.
#include "lnmod_ckpt_kernels.hpp"
#include "lnmod_code_shapes.hpp"
#include "lnmod_launch.hpp"

namespace lnmod {
namespace {

// f(element type, code)
template <typename F>
bool for_types(int dtype, int code, F&& f) {
    if (dtype == 0) return code == 0 ? f(bf16_io{}, int8_code{}) : f(bf16_io{}, e4m3_code{});
    return code == 0 ? f(f32_io{}, int8_code{}) : f(f32_io{}, e4m3_code{});
}

Codes codes_of(const Problem& p, const Checkpoint& c) {
    Codes cd;
    cd.codes = c.codes;
    cd.scales = c.scales;
    cd.lanes_log2 = group_lanes_log2(c.group);
    cd.groups = static_cast<int32_t>((p.D + c.group - 1) / c.group);
    cd.keep = keep_codes(p.T, p.D, 20000000, 70000000);
    return cd;
}

// Clusters of a forward launch on several segments: a block reloads its modulation registers once per segment of its
// cluster's region, and every further window costs bandwidth (see flat_clusters in lnmod_fwd.hip, whose rule this is).
int64_t fwd_clusters(int64_t nseg) {
    if (nseg <= 1) return 1;
    int64_t c = 2;
    while (c < 32 && nseg > 32 * c) c *= 2;
    return c;
}

// The waves that an entry puts into a block of rows of one wave fit the kernel's launch bounds.
template <typename Tag>
constexpr bool groups_fit(const ShapeTable& t) {
    for (const Shape& s : t)
        if (s.K == 1 && s.per_cu > groups_most(1, ckpt_bwd_waves(s.VPL, Unit<Tag>::NV, s.R, false))) return false;
    return true;
}
static_assert(groups_fit<bf16_io>(kCkptBwd50) && groups_fit<bf16_io>(kCkptBwdLong) && groups_fit<bf16_io>(kCkptBwdSegs) &&
              groups_fit<f32_io>(kCkptBwd50x32) && groups_fit<f32_io>(kCkptBwd32), "more waves than the kernel's launch bounds");

}  // namespace

RowPlan ckpt_bwd_plan(int64_t T, int64_t nseg, int64_t D, int dtype, Shape* shape, const Shape* force) {
    const Shape sh = pick_shape(force, ckpt_bwd_shape(T, nseg, static_cast<int>(D / kUnit), dtype));
    if (shape) *shape = sh;
    // a row moves 2 D elements (dy, dx) and D codes, a slot 2 D floats that are written and read back
    const double row = 2.0 * (dtype == 0 ? 2.0 : 4.0) + 1.0;
    const double stream_us = static_cast<double>(T) * static_cast<double>(D) * row / 5.8e6;
    return plan_rows_slots(T, nseg, group_blocks_most(sh), sh.R * row_groups(T, sh), stream_us, 16.0 / row, sh.clusters);
}

int64_t ckpt_bwd_most_slots(int64_t T, int64_t D, int dtype) {
    return T <= 0 ? 0 : most_slots(T, ckpt_bwd_shape(T, 1, static_cast<int>(D / kUnit), dtype));
}

hipError_t launch_ckpt_fwd(const Problem& p, bool token, const void* x, const void* shift, const void* scale, void* y,
                           const Checkpoint& c, int code, float* mean, float* rstd, hipStream_t st) {
    CkptFwdArgs a{};
    a.f.x = x;
    a.f.shift = shift;
    a.f.scale = scale;
    a.f.y = y;
    a.f.mean = mean;
    a.f.rstd = rstd;
    a.f.seg = Segments{p.cu, p.S, p.nseg};
    a.f.T = p.T;
    a.f.D = static_cast<int32_t>(p.D);
    a.f.nchunks = static_cast<int32_t>(p.D / kUnit);
    a.f.eps = p.eps;
    a.f.inv_D = 1.0f / static_cast<float>(p.D);
    a.c = codes_of(p, c);
    const Shape sh = pick_shape(p.force, token ? ckpt_tok_shape(p.T, a.f.nchunks, p.dtype, false)
                                             : ckpt_fwd_shape(p.T, p.nseg, a.f.nchunks, p.dtype));
    if (!covers(sh, a.f.nchunks)) return hipErrorInvalidConfiguration;
    const int groups = token ? 1 : fwd_row_groups(p.T, sh);
    const RowPlan pl = plan_rows_clusters(p.T, token ? 1 : p.nseg, static_cast<int64_t>(kNumCU) * sh.per_cu / groups, sh.R * groups,
                                          token ? 1 : fwd_clusters(p.nseg), sh.clusters);
    a.f.rows_per_cluster = pl.rows_per_cluster;
    a.f.nb = pl.nb;
    a.f.interleave = cluster_interleave(p.force, pl);
    a.f.split = cluster_split(a.f.interleave, pl);
    const dim3 grid(static_cast<unsigned>(pl.blocks)), block(sh.K * groups * kWave);
    const bool ok = for_types(p.dtype, code, [&](auto io, auto cd) {
        const auto go = [&](auto vpl, auto k, auto r, auto tok) {
            hipLaunchKernelGGL((ckpt_fwd_kernel<decltype(io), decltype(cd), vpl, k, r, tok>), grid, block, 0, st, a);
        };
        if (token) return ShapesOf<kSplit, kTokFwd>::call(sh, [&](auto... c) { go(c..., std::true_type{}); });
        const auto plain = [&](auto... c) { go(c..., std::false_type{}); };
        if constexpr (std::is_same<decltype(io), bf16_io>::value)
            return ShapesOf<kSplit, kCkptFwd40, kCkptFwd200, kCkptFwdLong, kCkptFwdSegs>::call(sh, plain);
        else
            return ShapesOf<kSplit, kCkptFwd32>::call(sh, plain);
    });
    return ok ? hipGetLastError() : hipErrorInvalidConfiguration;
}

hipError_t launch_ckpt_bwd(const Problem& p, bool token, const void* dy, const Checkpoint& c, int code, const void* scale,
                           const float* mean, const float* rstd, void* dx, void* dshift, void* dscale, bool io_grads,
                           float* ws, hipStream_t st) {
    CkptBwdArgs a{};
    a.b.dy = dy;
    a.b.scale = scale;
    a.b.mean = mean;
    a.b.rstd = rstd;
    a.b.dx = dx;
    a.b.dshift = token ? dshift : nullptr;
    a.b.dscale = token ? dscale : nullptr;
    a.b.ws = ws;
    a.b.seg = Segments{p.cu, p.S, p.nseg};
    a.b.T = p.T;
    a.b.D = static_cast<int32_t>(p.D);
    a.b.nchunks = static_cast<int32_t>(p.D / kUnit);
    a.b.inv_D = 1.0f / static_cast<float>(p.D);
    a.c = codes_of(p, c);
    Shape sh;
    RowPlan pl = ckpt_bwd_plan(p.T, p.nseg, p.D, p.dtype, &sh, p.force);
    if (token) {
        sh = pick_shape(p.force, ckpt_tok_shape(p.T, a.b.nchunks, p.dtype, true));
        pl = plan_rows(p.T, static_cast<int64_t>(kNumCU) * sh.per_cu, sh.R);
    }
    if (!covers(sh, a.b.nchunks)) return hipErrorInvalidConfiguration;
    a.b.rows_per_cluster = pl.rows_per_cluster;
    a.b.nb = pl.nb;
    a.b.interleave = cluster_interleave(p.force, pl);
    a.b.split = cluster_split(a.b.interleave, pl);
    const int groups = token ? 1 : row_groups(p.T, sh);
    bool fits = true;
    const dim3 grid(static_cast<unsigned>(pl.blocks)), block(sh.K * groups * kWave);
    const bool ok = for_types(p.dtype, code, [&](auto io, auto cd) {
        const auto go = [&](auto vpl, auto k, auto r, auto tok) {
            constexpr int waves = ckpt_bwd_waves(vpl, Unit<decltype(io)>::NV, r, tok);
            const size_t lds = group_lds(groups, units_at_once(vpl, waves), 2);
            fits = groups <= groups_most(k, waves);
            if (fits) hipLaunchKernelGGL((ckpt_bwd_kernel<decltype(io), decltype(cd), vpl, k, r, tok>), grid, block, lds, st, a);
        };
        if (token) return ShapesOf<kSplit, kTokBwdLong>::call(sh, [&](auto... c) { go(c..., std::true_type{}); });
        const auto plain = [&](auto... c) { go(c..., std::false_type{}); };
        if constexpr (std::is_same<decltype(io), bf16_io>::value)
            return ShapesOf<kCkptBwd50, kCkptBwdLong, kCkptBwdSegs>::call(sh, plain);
        else
            return ShapesOf<kCkptBwd50x32, kCkptBwd32>::call(sh, plain);
    });
    if (!ok || !fits) return hipErrorInvalidConfiguration;
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || token) return e;

    ReduceArgs r{};
    r.ws = ws;
    r.out[0] = dshift;
    r.out[1] = dscale;
    r.out_bf16 = io_grads && p.dtype == 0;
    r.seg = a.b.seg;
    r.T = p.T;
    r.rows_per_cluster = a.b.rows_per_cluster;
    r.nb = a.b.nb;
    r.D = a.b.D;
    r.nsum = 2;
    return launch_reduce(r, pl.clusters, st);
}

}  // namespace lnmod
