// lnmod_rotary.hip -- plan, instantiation and launch of the rotation and of the query and key norm with it.
#include <algorithm>

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

// Units of a lane that are compiled: a row of 8192 features by eight waves needs four, eight in fp32; where a lane keeps no
// weights' sums a row, backwards have three at most.
constexpr bool has_vpl(bool f32, int norm, int vpl, bool backward) {
    return vpl <= 3 || (vpl == 4 && (norm == kRowNorm || !backward)) || (f32 && norm == kRowNorm && vpl == 8);
}

template <template <typename, int, bool, int> class Go, typename Tag, int NORM, bool HALVES, int VPL>
bool one_vpl(const RotaryArgs& a, const RotaryShape& sh, hipStream_t st) {
    constexpr bool kBackward = std::is_same<Go<Tag, NORM, HALVES, VPL>, Bwd<Tag, NORM, HALVES, VPL>>::value;
    if constexpr (has_vpl(std::is_same<Tag, f32_io>::value, NORM, VPL, kBackward)) {
        if (sh.vpl != VPL) return false;
        const unsigned blocks = static_cast<unsigned>(a.side[0].blocks + a.side[1].blocks);
        Go<Tag, NORM, HALVES, VPL>::go(a, blocks, static_cast<unsigned>(sh.block_waves * kWave), st);
        return true;
    }
    return false;
}

template <template <typename, int, bool, int> class Go, typename Tag, int NORM, bool HALVES>
bool by_vpl(const RotaryArgs& a, const RotaryShape& sh, hipStream_t st) {
    return one_vpl<Go, Tag, NORM, HALVES, 1>(a, sh, st) || one_vpl<Go, Tag, NORM, HALVES, 2>(a, sh, st) ||
           one_vpl<Go, Tag, NORM, HALVES, 3>(a, sh, st) || one_vpl<Go, Tag, NORM, HALVES, 4>(a, sh, st) ||
           one_vpl<Go, Tag, NORM, HALVES, 8>(a, sh, st);
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

// Launch shapes, from sweeps of 1 to 4 units a lane, 1 to 8 waves a block and 1 to 128 blocks a CU over 73 problems (both types,
// 4 to 64 heads of 64 to 256 features, 1560 to 75 600 tokens).
//
// Three units a lane where nothing is against it: more loads in flight than with fewer, and registers for four waves a SIMD.
// Forwards four, where a round of heads is less idle so.  Backwards, where a CU holds eight waves, two or three, whichever
// leaves it fewer empty (of 28 heads of 128: 389 us with three units in three waves, 204 with two in four), and four where two
// waves have a row then (32 x 72: 243 us, 255 with fewer).
//
// Blocks forwards are what a CU holds at once where a norm over rows has its weights loaded (64 heads of 128: 203 us with four
// blocks a CU where three fit, 188 with three).  Else, and where blocks of three waves would have to be packed four to a CU,
// which they are after an idle moment (32 760 x 40 x 128: 238 us) but not while another kernel drains (316, with 32 blocks a CU
// 244), more of them even out the CUs (a row of four waves without a norm: two tokens side by side in a block of eight, 75 600 x
// 40 x 128 586 -> 550 us).
//
// Without a norm one block of six waves a CU is better still where the queries' rows are the keys' and three waves take a row, or
// fewer and no round of heads is idle: 75 600 x 40 x 128 540 -> 529 us, 6000 tokens of it 57 -> 47, 32 760 x 36 x 128 215 -> 204,
// 75 600 x 12 x 128 165 -> 160.  Not with idle rounds (20 heads: 146 and 150 us), nor with pairs of halves (24 x 128: 159 and 163).
//
// Backwards a block keeps its partial sums, and one for a CU is best: of eight waves where a row takes two or more (32 760 x 40 x 128
// 360 us in two blocks of four waves, 335 in one of eight), else of four (24 heads of 128, a norm for each: 258 us in two blocks
// of four waves, 245 in one), twice that where a lane has two units only.  Rows of different lengths, of queries and of
// keys, take three times as many blocks (28 and 4 heads: 235 -> 204 us).
RotaryShape shape_for(const RotaryArgs& a, bool halves, int norm, bool backward) {
    int rounds = 1;
    for (const RotarySide& s : a.side) {
        if (s.heads == 0) continue;
        const int r = head_split(s.heads, a.g_log2).rounds;
        if (r > rounds) rounds = r;
    }
    const auto waves_of = [&](int vpl) { return (rounds + vpl - 1) / vpl; };
    int vpl = 3;
    if (backward) {
        const auto held = [&](int vpl) { return 8 / waves_of(vpl) * waves_of(vpl); };
        if (held(2) > held(3) || (held(2) == held(3) && waves_of(2) * 2 < waves_of(3) * 3)) vpl = 2;
        if (norm == kRowNorm && rounds == 8) vpl = 4;
    } else if (waves_of(4) * 4 < waves_of(3) * 3 || (norm == kRowNorm && rounds > 6)) {
        vpl = 4;
    }
    if (vpl > rounds) vpl = rounds;
    if (norm == kRowNorm) {                                          // eight waves hold a row
        while (waves_of(vpl) > 8) vpl = vpl < 4 ? vpl + 1 : 8;
    }
    const bool even = a.side[0].heads == a.side[1].heads || a.side[1].heads == 0;
    if (norm == kNoNorm && even && !halves) {
        const int v = rounds > 9 && waves_of(4) == 3 ? 4 : vpl, k = waves_of(v);
        if (v >= 3 && (k == 3 || (6 % k == 0 && k * v == rounds))) return {v, 6, 1};
    }
    int waves = waves_of(vpl), per_cu = 32;
    if (waves > 8) waves = 8;
    if (backward && even && norm == kRowNorm && waves > 1) waves = 8 / waves * waves;
    else if (waves < 4) waves = waves * (4 / waves);
    else if (waves == 4 && norm == kNoNorm) waves = 8;
    if (backward) {
        per_cu = waves > 4 || (even && vpl >= 3) ? 1 : 2;
        if (!even) per_cu *= 3;
    } else if (norm == kRowNorm && waves != 3) {
        per_cu = std::max(1, (vpl <= 3 ? 16 : vpl == 4 ? 12 : 8) / waves);             // see LNMOD_OCCUPANCY
    }
    return {vpl, waves, per_cu};
}

}  // namespace

void rotary_bwd_slots(int dtype, int64_t N, const int32_t (&heads)[2], int head_dim, int norm, int64_t (&slots)[2]) {
    RotaryArgs a{};
    a.N = N;
    a.head_dim = head_dim;
    for (int t = 0; t < 2; ++t) a.side[t].heads = heads[t];
    lay_out(a, dtype);
    plan_rotary(a, shape_for(a, false, norm, true), norm != kRowNorm);
    for (int t = 0; t < 2; ++t) slots[t] = a.side[t].blocks;
}

hipError_t launch_rotary_fwd(int dtype, int norm, bool halves, RotaryArgs a, hipStream_t st) {
    lay_out(a, dtype);
    const RotaryShape sh = shape_for(a, halves, norm, false);
    plan_rotary(a, sh, norm != kRowNorm);
    a.sample_of = Divider(static_cast<uint32_t>(a.S));
    const bool ok = norm == kNoNorm    ? by_type<Fwd, kNoNorm>(dtype, halves, a, sh, st)
                    : norm == kRowNorm ? by_type<Fwd, kRowNorm>(dtype, halves, a, sh, st)
                                       : by_type<Fwd, kHeadNorm>(dtype, halves, a, sh, st);
    return ok ? hipGetLastError() : hipErrorInvalidConfiguration;
}

hipError_t launch_rotary_bwd(int dtype, int norm, bool halves, RotaryArgs a, void* const (&dw)[2], bool io_grads, float* ws,
                             hipStream_t st) {
    lay_out(a, dtype);
    const RotaryShape sh = shape_for(a, false, norm, true);
    plan_rotary(a, sh, norm != kRowNorm);
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
    const dim3 grid(static_cast<unsigned>((widest + kDwFeatures - 1) / kDwFeatures), 2);
    if (io_grads && dtype == 0) hipLaunchKernelGGL((rotary_dw_kernel<bf16_io>), grid, dim3(16 * kWave), 0, st, r);
    else hipLaunchKernelGGL((rotary_dw_kernel<f32_io>), grid, dim3(16 * kWave), 0, st, r);
    return hipGetLastError();
}

}  // namespace lnmod
