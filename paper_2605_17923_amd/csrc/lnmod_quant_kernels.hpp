// lnmod_quant_kernels.hpp -- gfx950 device code of the 8-bit checkpoint of a tensor and the way back (see lnmod_code.hpp for
// the codes).  Both move their bytes once and do little with them, so what bounds them is HBM: 3 (bf16) or 5 (fp32) bytes per
// feature.  The pattern is the plain copy's: a wave takes V pieces of 64 units (eight features a lane), the waves of the
// grid take consecutive pieces, and the next ones are requested before the current ones are computed.  A group is 4, 8
// or 16 lanes, so its largest magnitude needs two to four DPP steps and no LDS.  75 600 x 5120 bf16, groups of 128: 185 us, 6.3
// TB/s, and 192 us back, 6.1 TB/s, where a copy reaches 6.1.
//
// Rows whose length is a whole number of groups are one long row, cut into pieces of 64 units.  Otherwise (PAD) a piece can
// hold the end of one row and the start of others, and a lane finds its row by a comparison or a multiplication.  On the
// way back the units stay the long row that they are in memory; to quantise, every row is lengthened by idle units to a whole
// number of groups.  With pieces that end where the rows do, 75 600 x 200 bf16 took 22 us, now 12 and 10 back; 75 600 x 5000 takes
// 219 us and 188 back: the lengthened rows' pieces begin inside 128-byte lines.
#pragma once
#include "lnmod_code.hpp"
#include "lnmod_code_shapes.hpp"

namespace lnmod {

struct QuantArgs {
    void* x;                 // quantise: in;  dequantise: out
    void* codes;
    float* scales;
    int64_t rows;            // PAD: of the tensor;  else pieces
    int64_t total;           // units
    int64_t row_step;        // between two steps of a wave: rows (pieces) ...
    int32_t slot_step;       // ... and units
    int32_t units;           // of a row
    int32_t slots;           // PAD: units of a row, lengthened or not
    int32_t groups;          // of a row
    int32_t lanes_log2;      // of a group
    int32_t rows_in_64;      // 64 / slots and what is left
    int32_t left_in_64;
    uint32_t over_slots;     // PAD, slots < 64: ceil(65536 / slots), exact for what is divided (below 128)
    int32_t keep;            // see keep_codes
};

constexpr uint32_t kNoUnit = 0x03fffffeu;    // its offsets lie beyond every buffer here

template <typename Tag, typename C, int V, bool BACK, bool PAD>
__global__ __launch_bounds__(kQuantWaves* kWave) void quant_kernel(const QuantArgs a) {
    constexpr int NV = Unit<Tag>::NV;
    constexpr int64_t kMostRows = kWave + 1;                 // that a piece can touch
    const uint32_t lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool leads = (lane & ((1u << a.lanes_log2) - 1u)) == 0;

    // A piece: 64 units from unit `slot` of row `row` on (PAD), or the row-th 64 of all units.
    struct Piece {
        int64_t unit0, scale0;           // where its buffers start
        uint32_t units, scales;          // and end
        uint32_t unit, scale;            // the lane's, from there
    };
    const auto piece_at = [&](int64_t row, int32_t slot) {
        Piece p;
        if constexpr (PAD) {
            const int64_t left = a.rows - row;
            const uint32_t n = static_cast<uint32_t>(left < 0 ? 0 : left < kMostRows ? left : kMostRows);
            const uint32_t t = static_cast<uint32_t>(slot) + lane, slots = static_cast<uint32_t>(a.slots);
            const uint32_t k = slots >= kWave ? (t >= slots ? 1u : 0u) : (t * a.over_slots) >> 16;
            const uint32_t u = t - k * slots;
            p.unit0 = row * a.units;
            p.scale0 = row * a.groups;
            p.units = n * static_cast<uint32_t>(a.units);
            p.scales = n * static_cast<uint32_t>(a.groups);
            p.unit = u < static_cast<uint32_t>(a.units) ? k * static_cast<uint32_t>(a.units) + u : kNoUnit;
            p.scale = k * static_cast<uint32_t>(a.groups) + (u >> a.lanes_log2);
        } else {
            const int64_t left = a.total - row * kWave;
            p.unit0 = row * kWave;
            p.scale0 = p.unit0 >> a.lanes_log2;
            p.units = static_cast<uint32_t>(left < 0 ? 0 : left < kWave ? left : kWave);
            p.scales = p.units >> a.lanes_log2;              // whole groups
            p.unit = lane;
            p.scale = lane >> a.lanes_log2;
        }
        return p;
    };
    const auto x_of = [&](const Piece& p) { return row_of(a.x, p.unit0 * Unit<Tag>::kBytes, p.units * Unit<Tag>::kBytes); };
    const auto codes_of = [&](const Piece& p) { return row_of(a.codes, p.unit0 * 8, p.units * 8u); };
    const auto scales_of = [&](const Piece& p) { return row_of(a.scales, p.scale0 * 4, p.scales * 4u); };

    // the wave's V pieces from (row, slot) on
    struct Pieces {
        int64_t row[V];
        int32_t slot[V];
    };
    const auto pieces_from = [&](int64_t row, int32_t slot) {
        Pieces p;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            p.row[i] = row;
            p.slot[i] = slot;
            if constexpr (PAD) {
                row += a.rows_in_64;
                slot += a.left_in_64;
                if (slot >= a.slots) {
                    slot -= a.slots;
                    ++row;
                }
            } else {
                ++row;
            }
        }
        return p;
    };
    struct Step {
        u32x4 x[BACK ? 1 : V][NV];
        u32x2 code[BACK ? V : 1];
        float s[BACK ? V : 1];
    };
    const auto fetch = [&](const Pieces& at, Step& q) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const Piece p = piece_at(at.row[i], at.slot[i]);
            if constexpr (BACK) {
                q.code[i] = load_codes(codes_of(p), p.unit);
                q.s[i] = load_float(scales_of(p), p.scale * 4u);
            } else {
                load_unit<Tag>(x_of(p), p.unit, q.x[i]);
            }
        }
    };

    const int64_t first = (static_cast<int64_t>(blockIdx.x) * kQuantWaves + wave) * V;
    int64_t r = first;
    int32_t c = 0;
    if constexpr (PAD) {
        r = first * kWave / a.slots;
        c = static_cast<int32_t>(first * kWave - r * a.slots);
    }
    Pieces cur = pieces_from(r, c);
    Step now;
    fetch(cur, now);
    while (r < a.rows) {
        r += a.row_step;
        if constexpr (PAD) {
            c += a.slot_step;
            if (c >= a.slots) {
                c -= a.slots;
                ++r;
            }
        }
        const Pieces next = pieces_from(r, c);
        Step then;
        fetch(next, then);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const Piece p = piece_at(cur.row[i], cur.slot[i]);
            float v[8];
            if constexpr (BACK) {
                stand_for<Tag, C>(now.code[i], now.s[i], v);
                u32x4 o[NV];
                Unit<Tag>::pack(v, o);
                store_unit<Tag>(x_of(p), p.unit, o);
            } else {
                const Scale sc = scale_of<C>(group_max(Unit<Tag>::amax_bits(now.x[i]), a.lanes_log2));
                Unit<Tag>::unpack(now.x[i], v);
                store_codes(codes_of(p), p.unit, encode<C>(v, sc), a.keep);
                store_float(scales_of(p), leads ? p.scale * 4u : kNowhere, sc.s);
            }
        }
        cur = next;
        now = then;
    }
}

}  // namespace lnmod
