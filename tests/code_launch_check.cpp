// Host-side invariants of the launches of csrc/lnmod_code_shapes.hpp (compiled and run by test_code_launch_plan_cpu.py; no
// device code, no GPU).
#include <cstdint>
#include <cstdio>
#include <random>
#include "lnmod_code_shapes.hpp"

using namespace lnmod;

static int bad = 0;
#define CHECK(cond, ...) do { if (!(cond)) { if (bad < 20) { std::printf("FAIL %s: ", #cond); std::printf(__VA_ARGS__); std::printf("\n"); } ++bad; } } while (0)

static void check_shape(const char* which, int dtype, int units, const Shape& s) {
    CHECK(s.K >= 1 && s.K <= 16 && s.VPL >= 1 && s.VPL <= 6 && (s.R == 1 || s.R == 2), "%s dtype %d units %d: %d %d %d", which, dtype,
          units, s.K, s.VPL, s.R);
    CHECK(s.K * s.VPL * 64 >= units, "%s dtype %d units %d: %d x %d", which, dtype, units, s.K, s.VPL);
    CHECK(int64_t(kNumCU) * s.per_cu * s.K * 64 < (int64_t(1) << 32), "%s: a grid of too many threads", which);
    for (const int64_t T : {1, 1000, 5000, 500000}) {
        const int g = fwd_row_groups(T, s);
        CHECK(g == 1 || (g == kFwdGroups && s.K == 1 && s.per_cu >= g && T >= int64_t(kNumCU) * s.R * g), "%s T %lld: %d rows", which, (long long)T, g);
    }
}

// blocks whose waves hold rows of their own: every CU has one where the rows allow it, and never more waves than the entry says
static void check_rows(const char* which, int dtype, int units, int64_t T, const Shape& s) {
    check_shape(which, dtype, units, s);
    const int g = row_groups(T, s);
    CHECK(g >= 1 && (s.K > 1 ? g == 1 : g <= s.per_cu && g <= 12), "%s T %lld: %d rows", which, (long long)T, g);
    CHECK(s.K > 1 || g == 1 || (T + int64_t(s.R) * g - 1) / (s.R * g) * 2 >= kNumCU, "%s T %lld: CUs without a block", which, (long long)T);
    CHECK(group_blocks_most(s) * (s.K > 1 ? 1 : s.per_cu) == int64_t(kNumCU) * s.per_cu, "%s", which);
}

int main() {
    const int64_t rows[] = {1, 2, 3, 37, 500, 4099, 20000, 75600, 450000, (int64_t(1) << 31) - 1};
    for (int dtype = 0; dtype < 2; ++dtype)
        for (int units = 1; units <= 1024; ++units)
            for (const int64_t T : rows) {
                for (int64_t nseg = 1; nseg < 100; nseg += 40) {
                    check_shape("checkpoint forward", dtype, units, ckpt_fwd_shape(T, nseg, units, dtype));
                    check_rows("checkpoint backward", dtype, units, T, ckpt_bwd_shape(T, nseg, units, dtype));
                }
                for (const bool back : {false, true}) check_shape("per token", dtype, units, ckpt_tok_shape(T, units, dtype, back));
                check_shape("rms forward", dtype, units, rms_fwd_shape(T, units, dtype));
                for (const bool dh : {false, true}) check_rows("rms backward", dtype, units, T, rms_bwd_shape(T, units, dtype, dh));
            }
    // quantize and dequantize: from one piece to more than a card's memory holds; a grid of fewer than 2^32 threads whose blocks
    // all have a piece, and blocks for every piece unless the grid is at its largest
    std::mt19937_64 rng(5);
    for (int i = 0; i < 200000; ++i) {
        const int64_t pieces = 1 + static_cast<int64_t>(rng() % (uint64_t(1) << (rng() % 31)));
        const int dtype = static_cast<int>(rng() % 2);
        const QuantShape sh = quant_shape(pieces * 512 * (dtype == 0 ? 2 : 4), dtype);
        const int64_t blocks = quant_blocks(pieces, sh), per_block = int64_t(kQuantWaves) * sh.pieces;
        CHECK(blocks >= 1 && blocks * kQuantWaves * 64 < (int64_t(1) << 32), "dtype %d, %lld pieces: %lld blocks", dtype,
              (long long)pieces, (long long)blocks);
        CHECK((blocks - 1) * per_block < pieces, "dtype %d, %lld pieces: an idle block", dtype, (long long)pieces);
        CHECK(blocks * per_block >= pieces || blocks == int64_t(kNumCU) * sh.per_cu, "dtype %d, %lld pieces: %lld blocks", dtype,
              (long long)pieces, (long long)blocks);
    }
    std::printf("%d failures\n", bad);
    return bad != 0;
}
