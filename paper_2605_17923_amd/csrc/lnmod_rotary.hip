// lnmod_rotary.hip -- plan, instantiation and launch of the rotation and of the query and key norm with it.
#include "lnmod_rotary_kernels.hpp"

namespace lnmod {
namespace {

template <typename Tag, int NORM, bool HALVES, int VPL>
struct Fwd {
    static void go(const RotaryArgs& a, unsigned blocks, unsigned threads, hipStream_t st) {
        hipLaunchKernelGGL((rotary_fwd_kernel<Tag, NORM, HALVES, VPL>), dim3(blocks), dim3(threads), 0, st, a);
    }
};
template <typename Tag, int NORM, bool HALVES, int VPL>
struct Bwd {
    static void go(const RotaryArgs& a, unsigned blocks, unsigned threads, hipStream_t st) {
        size_t lds = 0;
        for (const RotarySide& s : a.side) {
            const int turns = NORM == kRowNorm ? s.teams : s.teams * s.waves;
            if (turns > 1 && lds < s.width * sizeof(float)) lds = s.width * sizeof(float);
        }
        hipLaunchKernelGGL((rotary_bwd_kernel<Tag, NORM, HALVES, VPL>), dim3(blocks), dim3(threads), lds, st, a);
    }
};

template <template <typename, int, bool, int> class Go, typename Tag, int NORM, bool HALVES>
bool by_vpl(const RotaryArgs& a, const RotaryShape& sh, hipStream_t st) {
    const unsigned blocks = static_cast<unsigned>(a.side[0].blocks + a.side[1].blocks);
    const unsigned threads = static_cast<unsigned>(sh.block_waves * kWave);
    switch (sh.vpl) {
        case 1: Go<Tag, NORM, HALVES, 1>::go(a, blocks, threads, st); return true;
        case 2: Go<Tag, NORM, HALVES, 2>::go(a, blocks, threads, st); return true;
        case 3: Go<Tag, NORM, HALVES, 3>::go(a, blocks, threads, st); return true;
        case 4: Go<Tag, NORM, HALVES, 4>::go(a, blocks, threads, st); return true;
        default: break;
    }
    if constexpr (std::is_same<Tag, f32_io>::value && NORM == kRowNorm) {
        if (sh.vpl == 8) {
            Go<Tag, NORM, HALVES, 8>::go(a, blocks, threads, st);
            return true;
        }
    }
    return false;
}

template <template <typename, int, bool, int> class Go, int NORM>
bool by_type(int dtype, bool halves, const RotaryArgs& a, const RotaryShape& sh, hipStream_t st) {
    if (dtype == 0) return halves ? by_vpl<Go, bf16_io, NORM, true>(a, sh, st) : by_vpl<Go, bf16_io, NORM, false>(a, sh, st);
    return halves ? by_vpl<Go, f32_io, NORM, true>(a, sh, st) : by_vpl<Go, f32_io, NORM, false>(a, sh, st);
}

void lay_out(RotaryArgs& a, int dtype) {
    a.units = a.head_dim / (dtype == 0 ? 8 : 4);
    a.g_log2 = ceil_log2(a.units);
}

RotaryShape shape_for(const RotaryArgs& a, int dtype, int norm, bool backward) {
    const int32_t heads[2] = {a.side[0].heads, a.side[1].heads};
    return rotary_shape(dtype, heads, a.g_log2, norm, backward);
}

}  // namespace

RotaryShape rotary_shape(int dtype, const int32_t (&heads)[2], int g_log2, int norm, bool backward) {
    int rounds = 1;
    for (const int32_t h : heads) {
        if (h == 0) continue;
        const int r = head_split(h, g_log2).rounds;
        if (r > rounds) rounds = r;
    }
    (void)backward;
    int vpl = rounds <= 8 ? (rounds + 3) / 4 : rounds <= 16 ? 2 : rounds <= 24 ? 3 : 4;
    if (dtype == 1 && norm == kRowNorm && rounds > 32) vpl = 8;
    int waves = (rounds + vpl - 1) / vpl;
    if (waves > 8) waves = 8;
    if (waves < 4) waves = waves * (4 / waves);
    return {vpl, waves};
}

int64_t rotary_blocks_per_cu(int norm, bool backward) {
    (void)norm;
    return backward ? 2 : 16;
}

void rotary_bwd_slots(int dtype, int64_t N, const int32_t (&heads)[2], int head_dim, int norm, int64_t (&slots)[2]) {
    RotaryArgs a{};
    a.N = N;
    a.head_dim = head_dim;
    for (int t = 0; t < 2; ++t) a.side[t].heads = heads[t];
    lay_out(a, dtype);
    plan_rotary(a, shape_for(a, dtype, norm, true), norm != kRowNorm, rotary_blocks_per_cu(norm, true));
    for (int t = 0; t < 2; ++t) slots[t] = a.side[t].blocks;
}

hipError_t launch_rotary_fwd(int dtype, int norm, bool halves, RotaryArgs a, hipStream_t st) {
    lay_out(a, dtype);
    const RotaryShape sh = shape_for(a, dtype, norm, false);
    plan_rotary(a, sh, norm != kRowNorm, rotary_blocks_per_cu(norm, false));
    a.sample_of = Divider(static_cast<uint32_t>(a.S));
    const bool ok = norm == kNoNorm    ? by_type<Fwd, kNoNorm>(dtype, halves, a, sh, st)
                    : norm == kRowNorm ? by_type<Fwd, kRowNorm>(dtype, halves, a, sh, st)
                                       : by_type<Fwd, kHeadNorm>(dtype, halves, a, sh, st);
    return ok ? hipGetLastError() : hipErrorInvalidConfiguration;
}

hipError_t launch_rotary_bwd(int dtype, int norm, bool halves, RotaryArgs a, void* const (&dw)[2], bool io_grads, float* ws,
                             hipStream_t st) {
    lay_out(a, dtype);
    const RotaryShape sh = shape_for(a, dtype, norm, true);
    plan_rotary(a, sh, norm != kRowNorm, rotary_blocks_per_cu(norm, true));
    a.sample_of = Divider(static_cast<uint32_t>(a.S));
    RotaryDwArgs r{};
    int widest = 0;
    for (int t = 0; t < 2; ++t) {
        RotarySide& s = a.side[t];
        s.ws = ws;
        r.ws[t] = ws;
        r.dw[t] = dw[t];
        r.slots[t] = s.blocks;
        r.width[t] = s.width;
        if (s.width > widest) widest = s.width;
        ws += static_cast<int64_t>(s.blocks) * s.width;
    }
    const bool ok = norm == kRowNorm ? by_type<Bwd, kRowNorm>(dtype, halves, a, sh, st) : by_type<Bwd, kHeadNorm>(dtype, halves, a, sh, st);
    if (!ok) return hipErrorInvalidConfiguration;
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const dim3 grid(static_cast<unsigned>((widest + kWave - 1) / kWave), 2);
    if (io_grads && dtype == 0) hipLaunchKernelGGL((rotary_dw_kernel<bf16_io>), grid, dim3(16 * kWave), 0, st, r);
    else hipLaunchKernelGGL((rotary_dw_kernel<f32_io>), grid, dim3(16 * kWave), 0, st, r);
    return hipGetLastError();
}

}  // namespace lnmod
