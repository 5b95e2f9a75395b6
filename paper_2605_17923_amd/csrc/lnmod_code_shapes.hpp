// lnmod_code_shapes.hpp -- launch shapes {waves per row, units per lane, rows per block and step, blocks per CU} of the row
// kernels that hold activations in 8 bits, and their dispatch.
//
// A table has an entry per 512 features (one unit of eight features for each lane of one wave).  The entries are from a sweep of
// every (waves, units) that cover a row closely with one and two rows, 1 to 128 blocks per CU, at a multiple of 512 features and
// 200 below it, on x of 3, 20, 60, 120 and 500 MB, bf16 and fp32.  What they share: waves * units is the row's length in
// units of 512 features wherever that is possible, because every idle lane costs arithmetic, and the arithmetic of the
// few waves that HBM likes best is what limits them; forwards, which keep nothing from row to row but the weights, win with
// many more blocks than are resident (root-mean-square norm, 32 760 x 5120 bf16: 118 us with one block per CU, 80.5 with 64);
// backwards keep a slot of partial sums per block and stay at what is resident.  On short rows a backward's row belongs to one
// wave and a block is several of those (K = 1; "blocks per CU" are its waves): checkpoint bf16 up to five units a lane, six on
// more than 50 MB, fp32 two; rms norm bf16 three up to 50 MB, then one, two and five (three without a residual's gradient),
// fp32 one up to 50 MB, then three.  That needs no barrier in the loop, a slot per CU, and no luck with where the dispatcher
// puts blocks of one wave: checkpoint backward, 32 552 x 1536 bf16 57 us with three blocks of three waves per row, 51 with one of
// four; 130 208 x 1536 205 and 168; 78 125 x 2560 191 and 172.
// The classes of x's size and what the entries lose against the best shape of each problem, in the mean and at worst:
//   checkpoint forward   bf16 up to 10 MB 1.6 %, 5 %; 40 MB 2 %, 14 %; 200 MB 1 %, 6 %; beyond 1 %, 5 %;  fp32 1 to 3 %
//   rms norm forward     bf16 1 to 3 %, 14 %;  fp32 2 to 4 %
//   backwards            checkpoint 1 to 3 %, 8 % (3584 features 15 %), rms norm 1 to 3 %, 10 %
#pragma once
#include <array>
#include <utility>

#include "lnmod_launch.hpp"

namespace lnmod {

using ShapeTable = std::array<Shape, 16>;            // [k]: rows of more than 512 k and at most 512 (k + 1) features

constexpr bool covers_all(const ShapeTable& t) {
    for (int k = 0; k < 16; ++k)
        if (t[k].K * t[k].VPL < k + 1) return false;
    return true;
}
constexpr ShapeTable with(ShapeTable t, int rows, int per_cu) {
    for (int k = 0; k < 16; ++k) {
        t[k].R = rows;
        t[k].per_cu = per_cu;
    }
    return t;
}

// The split of a row that most kernels share.
inline constexpr ShapeTable kSplit = {{
    {1, 1, 1, 16}, {2, 1, 1, 16}, {3, 1, 1, 16}, {4, 1, 1, 16}, {5, 1, 1, 16}, {3, 2, 1, 16}, {4, 2, 1, 16}, {4, 2, 1, 16},
    {3, 3, 1, 16}, {5, 2, 1, 16}, {4, 3, 1, 16}, {4, 3, 1, 16}, {8, 2, 1, 16}, {8, 2, 1, 16}, {8, 2, 1, 16}, {8, 2, 1, 16}}};

// Checkpoint forward
inline constexpr ShapeTable kCkptFwd40 = {{
    {1, 1, 2, 16}, {1, 2, 2, 12}, {1, 3, 2, 8}, {1, 4, 2, 12}, {1, 5, 1, 12}, {3, 2, 2, 4}, {4, 2, 2, 4}, {4, 2, 2, 4},
    {3, 3, 1, 4}, {5, 2, 2, 2}, {4, 3, 2, 3}, {4, 3, 2, 3}, {4, 4, 2, 2}, {4, 4, 2, 2}, {4, 4, 2, 2}, {4, 4, 1, 2}}};
inline constexpr ShapeTable kCkptFwd200 = {{
    {1, 1, 2, 128}, {1, 2, 2, 64}, {1, 3, 2, 64}, {1, 4, 1, 4}, {1, 5, 1, 4}, {1, 6, 1, 4}, {4, 2, 1, 2}, {4, 2, 2, 64},
    {3, 3, 2, 128}, {5, 2, 1, 2}, {4, 3, 1, 1}, {4, 3, 1, 1}, {8, 2, 1, 1}, {8, 2, 1, 1}, {8, 2, 1, 1}, {4, 4, 1, 1}}};
inline constexpr ShapeTable kCkptFwdLong = {{
    {1, 1, 2, 128}, {1, 2, 2, 4}, {1, 3, 2, 4}, {4, 1, 2, 128}, {1, 5, 1, 4}, {3, 2, 2, 128}, {4, 2, 2, 128}, {4, 2, 2, 1},
    {3, 3, 2, 128}, {5, 2, 1, 64}, {4, 3, 2, 1}, {4, 3, 1, 1}, {4, 4, 1, 64}, {4, 4, 1, 1}, {8, 2, 2, 1}, {8, 2, 2, 1}}};
// several samples or segments, x beyond 40 MB: a block of few rows meets few segments, so two rows and as many blocks as they
// give (24 segments, 39 062 x 5120: 211 us with the entry above, 175; 96 segments 236 and 175)
inline constexpr ShapeTable kCkptFwdSegs = [] {
    ShapeTable t = with(kSplit, 2, 128);
    t[1] = {1, 2, 2, 128};
    t[2] = {1, 3, 2, 128};
    t[4] = {1, 5, 2, 128};
    t[9] = {4, 3, 2, 128};
    return t;
}();
inline constexpr ShapeTable kCkptFwd32 = {{
    {1, 1, 2, 8}, {1, 2, 2, 4}, {3, 1, 2, 3}, {1, 4, 1, 4}, {1, 5, 1, 4}, {3, 2, 1, 2}, {4, 2, 1, 2}, {4, 2, 1, 2},
    {3, 3, 1, 2}, {5, 2, 1, 1}, {4, 3, 1, 1}, {4, 3, 1, 1}, {4, 4, 1, 1}, {8, 2, 1, 1}, {4, 4, 1, 1}, {4, 4, 1, 1}}};

// Modulation rows per token: neither direction keeps anything from row to row, so both take many blocks; the backward on
// more than 200 MB has entries of its own.  2 to 5 % (forward) and 3 to 8 % off the best shape of each problem.
inline constexpr ShapeTable kTokBwd200 = with(kSplit, 1, 128);
inline constexpr ShapeTable kTokFwd = [] {
    ShapeTable t = with(kSplit, 1, 128);
    t[9].per_cu = 64;
    for (int k = 12; k < 16; ++k) t[k] = {4, 4, 1, 128};
    return t;
}();
inline constexpr ShapeTable kTokBwdLong = {{
    {1, 1, 2, 4}, {2, 1, 2, 2}, {3, 1, 2, 1}, {4, 1, 2, 128}, {5, 1, 2, 64}, {3, 2, 1, 1}, {4, 2, 1, 1}, {8, 1, 2, 64},
    {3, 3, 2, 64}, {5, 2, 1, 1}, {4, 3, 2, 1}, {4, 3, 1, 1}, {8, 2, 1, 1}, {8, 2, 1, 1}, {8, 2, 2, 1}, {8, 2, 1, 1}}};

// Root-mean-square norm, forward
inline constexpr ShapeTable kRmsFwd200 = [] {
    ShapeTable t = with(kSplit, 1, 128);
    for (int k = 1; k < 5; ++k) t[k] = {1, k + 1, 1, k < 4 ? 128 : 64};
    return t;
}();
inline constexpr ShapeTable kRmsFwdLong = [] {
    ShapeTable t = with(kSplit, 2, 128);
    t[1] = {1, 3, 2, 128};
    t[4] = {1, 5, 2, 128};
    return t;
}();
inline constexpr ShapeTable kRmsFwd32 = {{
    {1, 1, 2, 4}, {1, 2, 2, 4}, {1, 3, 1, 4}, {1, 4, 1, 4}, {1, 5, 1, 4}, {3, 2, 1, 2}, {4, 2, 1, 2}, {4, 2, 1, 2},
    {3, 3, 1, 2}, {5, 2, 1, 2}, {4, 3, 1, 1}, {4, 3, 1, 1}, {4, 4, 1, 1}, {4, 4, 1, 1}, {4, 4, 1, 1}, {4, 4, 1, 1}}};

// Backward from a checkpoint
inline constexpr ShapeTable kCkptBwd50 = {{
    {1, 1, 1, 12}, {1, 2, 2, 4}, {1, 3, 1, 4}, {1, 4, 1, 4}, {1, 5, 1, 3}, {3, 2, 2, 1}, {4, 2, 2, 1}, {4, 2, 2, 1},
    {3, 3, 2, 1}, {10, 1, 2, 1}, {12, 1, 2, 1}, {12, 1, 2, 1}, {8, 2, 2, 1}, {8, 2, 2, 1}, {8, 2, 2, 1}, {8, 2, 2, 1}}};
inline constexpr ShapeTable kCkptBwdLong = {{
    {1, 1, 2, 12}, {1, 2, 2, 4}, {1, 3, 1, 4}, {1, 4, 2, 3}, {1, 5, 1, 4}, {1, 6, 1, 4}, {4, 2, 2, 1}, {4, 2, 2, 1},
    {3, 3, 2, 1}, {4, 3, 2, 1}, {4, 3, 1, 1}, {4, 3, 1, 1}, {4, 4, 1, 1}, {4, 4, 1, 1}, {4, 4, 1, 1}, {4, 4, 1, 1}}};
// several samples or segments: 58 794 x 2048 in 40 of them, both passes, 250 us with {4, 1, 2, 2}, 231 (19 959 in 40 shorter ones 1 % more).
// Only this width was measured with segments; the others keep the entries of one sample.
inline constexpr ShapeTable kCkptBwdSegs = [] {
    ShapeTable t = kCkptBwdLong;
    t[3] = {1, 4, 1, 4};
    return t;
}();
inline constexpr ShapeTable kCkptBwd50x32 = {{
    {1, 1, 1, 8}, {1, 2, 1, 4}, {3, 1, 2, 1}, {4, 1, 2, 1}, {3, 2, 2, 1}, {3, 2, 2, 1}, {4, 2, 2, 1}, {4, 2, 2, 1},
    {3, 3, 2, 1}, {10, 1, 2, 1}, {12, 1, 2, 1}, {12, 1, 2, 1}, {8, 2, 1, 1}, {8, 2, 1, 1}, {8, 2, 1, 1}, {4, 4, 1, 1}}};
inline constexpr ShapeTable kCkptBwd32 = {{
    {1, 1, 2, 4}, {1, 2, 2, 3}, {5, 1, 2, 1}, {4, 1, 2, 1}, {3, 2, 2, 1}, {3, 2, 2, 1}, {4, 2, 2, 1}, {4, 2, 2, 1},
    {3, 3, 2, 1}, {4, 3, 1, 1}, {4, 3, 1, 1}, {4, 3, 1, 1}, {4, 4, 1, 1}, {4, 4, 1, 1}, {4, 4, 1, 1}, {4, 4, 1, 1}}};

// Root-mean-square norm, backward
inline constexpr ShapeTable kRmsBwd50 = {{
    {1, 1, 1, 12}, {1, 2, 1, 4}, {1, 3, 1, 3}, {4, 1, 2, 1}, {5, 1, 1, 1}, {6, 1, 1, 1}, {4, 2, 1, 1}, {8, 1, 2, 1},
    {10, 1, 2, 1}, {10, 1, 2, 1}, {12, 1, 2, 1}, {12, 1, 2, 1}, {8, 2, 2, 1}, {8, 2, 2, 1}, {8, 2, 2, 1}, {8, 2, 2, 1}}};
inline constexpr ShapeTable kRmsBwdLong = {{
    {1, 1, 2, 8}, {1, 2, 1, 4}, {3, 1, 2, 1}, {4, 1, 2, 1}, {1, 5, 1, 2}, {3, 2, 1, 1}, {3, 3, 1, 1}, {8, 1, 2, 1},
    {3, 3, 2, 1}, {10, 1, 1, 1}, {12, 1, 1, 1}, {12, 1, 1, 1}, {8, 2, 1, 1}, {4, 4, 1, 1}, {4, 4, 1, 1}, {8, 2, 1, 1}}};
// without a gradient along the residual stream: 32 552 x 1536 60.2 us with the entry above, 54.7.  Only this width was measured
// without one; the others keep the entries of the sweep with it.
inline constexpr ShapeTable kRmsBwdLongAlone = [] {
    ShapeTable t = kRmsBwdLong;
    t[2] = {1, 3, 1, 3};
    return t;
}();
inline constexpr ShapeTable kRmsBwd50x32 = {{
    {1, 1, 2, 3}, {3, 1, 1, 1}, {3, 1, 1, 1}, {4, 1, 1, 1}, {5, 1, 2, 1}, {3, 2, 1, 1}, {4, 2, 1, 1}, {4, 2, 1, 1},
    {3, 3, 1, 1}, {10, 1, 1, 1}, {4, 3, 1, 1}, {4, 3, 1, 1}, {8, 2, 1, 1}, {8, 2, 1, 1}, {4, 4, 1, 1}, {4, 4, 1, 1}}};
inline constexpr ShapeTable kRmsBwd32 = {{
    {1, 1, 2, 3}, {1, 2, 1, 3}, {1, 3, 2, 2}, {4, 1, 2, 1}, {3, 2, 2, 1}, {3, 2, 2, 1}, {4, 2, 2, 1}, {4, 2, 2, 1},
    {3, 3, 2, 1}, {4, 3, 2, 1}, {4, 3, 1, 1}, {4, 3, 1, 1}, {4, 4, 1, 1}, {4, 4, 1, 1}, {4, 4, 1, 1}, {4, 4, 1, 1}}};

static_assert(covers_all(kSplit) && covers_all(kCkptFwd40) && covers_all(kCkptFwd200) && covers_all(kCkptFwdLong) &&
              covers_all(kCkptFwd32) && covers_all(kCkptFwdSegs) && covers_all(kTokFwd) && covers_all(kTokBwd200) &&
              covers_all(kTokBwdLong) && covers_all(kRmsFwd200) && covers_all(kRmsFwdLong) && covers_all(kRmsFwd32) &&
              covers_all(kCkptBwd50) && covers_all(kCkptBwdLong) && covers_all(kCkptBwdSegs) && covers_all(kCkptBwd50x32) &&
              covers_all(kCkptBwd32) && covers_all(kRmsBwd50) && covers_all(kRmsBwdLong) && covers_all(kRmsBwdLongAlone) &&
              covers_all(kRmsBwd50x32) && covers_all(kRmsBwd32), "an entry that does not cover its rows");

inline const Shape& entry(const ShapeTable& t, int units) { return t[(units - 1) / 64]; }

inline Shape ckpt_fwd_shape(int64_t T, int64_t nseg, int units, int dtype) {
    const int64_t bytes = T * units * (dtype == 0 ? 16 : 32);
    if (bytes <= 10000000) return entry(kSplit, units);
    if (dtype != 0) return entry(kCkptFwd32, units);
    if (nseg > 1 && bytes > 40000000) return entry(kCkptFwdSegs, units);
    return entry(bytes <= 40000000 ? kCkptFwd40 : bytes <= 200000000 ? kCkptFwd200 : kCkptFwdLong, units);
}
inline Shape ckpt_tok_shape(int64_t T, int units, int dtype, bool backward) {
    const int64_t bytes = T * units * (dtype == 0 ? 16 : 32);
    if (bytes <= 10000000) return entry(kSplit, units);
    if (!backward) return entry(kTokFwd, units);
    return entry(bytes > 200000000 ? kTokBwdLong : kTokBwd200, units);
}
inline Shape rms_fwd_shape(int64_t N, int units, int dtype) {
    const int64_t bytes = N * units * (dtype == 0 ? 16 : 32);
    if (bytes <= 10000000) return entry(kSplit, units);
    if (dtype != 0) return entry(kRmsFwd32, units);
    return entry(bytes <= 200000000 ? kRmsFwd200 : kRmsFwdLong, units);
}
inline Shape ckpt_bwd_shape(int64_t T, int64_t nseg, int units, int dtype) {
    const bool shorter = T * units * (dtype == 0 ? 16 : 32) <= 50000000;
    if (dtype == 0) return entry(shorter ? kCkptBwd50 : nseg > 1 ? kCkptBwdSegs : kCkptBwdLong, units);
    return entry(shorter ? kCkptBwd50x32 : kCkptBwd32, units);
}
inline Shape rms_bwd_shape(int64_t N, int units, int dtype, bool dh) {
    const bool shorter = N * units * (dtype == 0 ? 16 : 32) <= 50000000;
    if (dtype == 0) return entry(shorter ? kRmsBwd50 : dh ? kRmsBwdLong : kRmsBwdLongAlone, units);
    return entry(shorter ? kRmsBwd50x32 : kRmsBwd32, units);
}

// Checkpoint of a tensor and the way back: pieces of 64 units that a wave takes per step, and blocks per CU that the grid has
// at most (many more than are resident: with four, 75 600 x 5120 bf16 took 211 us there and 217 back, with 64 it takes 187 and
// 194; 10 000 x 5120 30.8 and 31.4, with 32 of two pieces 26.7 and 27.4).  Small launches take one piece a wave, so that
// every CU has a part (200 x 5120 3.9 -> 2.7 us, 1025 x 1432 4.3 -> 3.3); fp32 units are 32 bytes of a lane and always take
// one, with a block for every four as long as a grid may have that many (20 000 x 5120 97 and 134 -> 88 and 95).
struct QuantShape {
    int pieces, per_cu;
};
constexpr int kQuantWaves = 4;
constexpr QuantShape kQuantWide = {1, 1 << 15};
static_assert(int64_t(kNumCU) * kQuantWide.per_cu * kQuantWaves * 64 < (int64_t(1) << 32), "a grid has fewer than 2^32 threads");

inline QuantShape quant_shape(int64_t bytes, int dtype) {
    if (dtype != 0) return kQuantWide;
    if (bytes <= 16000000) return {1, 16};
    return bytes <= 300000000 ? QuantShape{2, 32} : QuantShape{4, 64};
}
inline int64_t quant_blocks(int64_t pieces, const QuantShape& sh) {
    const int64_t per_block = int64_t(kQuantWaves) * sh.pieces, most = int64_t(kNumCU) * sh.per_cu;
    const int64_t blocks = (pieces + per_block - 1) / per_block;
    return blocks < most ? blocks : most;
}

// Waves of a backward block that hold rows of their own (K = 1: the entry's blocks per CU are the waves of one block, fewer
// where the rows give the CUs fewer).  Rounded up, so that every row is in work at once as far as the entry allows: just
// beyond a multiple of 256 R rows that leaves up to half of the CUs without a block (257 rows: 129 blocks), and is still the
// faster side.  Rounded down, which gives every CU a block and some waves a second row, both passes (us): checkpoint
// 300 x 1536 bf16 7.7 -> 8.5, 300 x 2560 9.4 -> 10.5, 640 x 2560 10.9 -> 11.7; rms norm 300 x 1536 6.2 -> 6.9; from 1024
// rows on the same.  So the blocks fall as the rows pass such a line, and the workspace queries ask for most_slots.
inline int row_groups(int64_t T, const Shape& sh) {
    if (sh.K > 1) return 1;
    const int64_t all = int64_t(kNumCU) * sh.R, g = (T + all - 1) / all;
    return g < 1 ? 1 : g < sh.per_cu ? static_cast<int>(g) : sh.per_cu;
}
inline int64_t group_blocks_most(const Shape& sh) { return int64_t(kNumCU) * (sh.K > 1 ? sh.per_cu : 1); }
// Slots of one sample's backward at most: what row_groups makes of T rows or fewer, which does not fall as T grows.
inline int64_t most_slots(int64_t T, const Shape& sh) { return grid_blocks(T, group_blocks_most(sh), sh.R); }

// The same in a forward, which has nothing to add: blocks of four waves with rows of their own in place of blocks of one
// (checkpoint forward 32 552 x 1536 bf16 5 % less than with three waves per row, rms norm 19 531 x 2560 without a residual 27 %).
constexpr int kFwdGroups = 4;
inline int fwd_row_groups(int64_t T, const Shape& sh) {
    return sh.K == 1 && sh.per_cu >= kFwdGroups && T >= int64_t(kNumCU) * sh.R * kFwdGroups ? kFwdGroups : 1;
}

// f(units per lane, waves, rows) as constants for the entry of one of the tables that sh is; false if it is none.  Only what
// the tables hold is compiled.
template <const ShapeTable&... TABS>
struct ShapesOf {
    template <typename F>
    static bool call(const Shape& sh, F&& f) {
        return (one<TABS>(sh, f, std::make_index_sequence<16>{}) || ...);
    }

private:
    template <const ShapeTable& TAB, typename F, size_t... I>
    static bool one(const Shape& sh, F&& f, std::index_sequence<I...>) {
        return (entry<TAB, I>(sh, f) || ...);
    }
    template <const ShapeTable& TAB, size_t I, typename F>
    static bool entry(const Shape& sh, F&& f) {
        using std::integral_constant;
        if (sh.K != TAB[I].K || sh.VPL != TAB[I].VPL || sh.R != TAB[I].R) return false;
        f(integral_constant<int, TAB[I].VPL>{}, integral_constant<int, TAB[I].K>{}, integral_constant<int, TAB[I].R>{});
        return true;
    }
};

}  // namespace lnmod
