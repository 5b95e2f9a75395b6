// lnmod_quant_kernels.hpp -- gfx950 device code of the 8-bit checkpoint of a tensor and the way back (see lnmod_code.hpp for
// the codes).  Both move their bytes once and do little with them, so what bounds them is HBM: 3 (bf16) or 5 (fp32) bytes per
// feature.  The pattern is the plain copy's: a wave takes V pieces of 64 units (eight features a lane), the waves of the
// grid take consecutive pieces, and the next ones are requested before the current ones are computed.  A group is 4, 8
// or 16 lanes, so its largest magnitude needs two to four DPP steps and no LDS.  75 600 x 5120 bf16, groups of 128: 189 us, 6.2
// TB/s, and 195 us back, 6.0 TB/s, where a copy reaches 6.1.
//
// Rows whose length is a whole number of groups are one long row, cut into pieces of 64 units; otherwise every row is cut
// into pieces of its own, and the last one has idle lanes.
#pragma once
#include "lnmod_code.hpp"
#include "lnmod_code_shapes.hpp"

namespace lnmod {

struct QuantArgs {
    void* x;                 // quantise: in;  dequantise: out
    void* codes;
    float* scales;
    int64_t rows;            // of `units` units (one long row: of 64, the last one shorter)
    int64_t total;           // units
    int32_t units;           // of a row
    int32_t per_row;         // pieces of a row
    int32_t groups;          // of a row
    int32_t lanes_log2;      // of a group
    int32_t keep;            // see keep_codes
    int64_t row_step;        // rows and pieces that lie between two steps of a wave
    int32_t piece_step;
};

// Where a wave is: V consecutive pieces from (row, piece) on.
template <int V>
struct Pieces {
    int64_t row[V];
    int32_t col[V];          // piece of its row
    __device__ inline void set(int64_t r, int32_t c, int32_t per_row) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            row[i] = r;
            col[i] = c;
            if (++c == per_row) {
                c = 0;
                ++r;
            }
        }
    }
};

template <typename Tag, typename C, int V, bool BACK>
__global__ __launch_bounds__(kQuantWaves* kWave) void quant_kernel(const QuantArgs a) {
    constexpr int NV = Unit<Tag>::NV;
    const uint32_t lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t first = (static_cast<int64_t>(blockIdx.x) * kQuantWaves + wave) * V;
    int64_t r = first / a.per_row;
    int32_t c = static_cast<int32_t>(first - r * a.per_row);

    struct Step {
        u32x4 x[V][BACK ? 1 : NV];
        u32x2 code[BACK ? V : 1];
        float s[BACK ? V : 1];
    };
    // units of piece i, 0 beyond the last row
    const auto units_at = [&](const Pieces<V>& p, int i) -> uint32_t {
        if (p.row[i] >= a.rows) return 0;
        const int64_t left = a.total - (p.row[i] * a.units + static_cast<int64_t>(p.col[i]) * kWave);
        const int32_t of_row = a.units - p.col[i] * kWave;
        const int64_t n = left < of_row ? left : of_row;
        return n < kWave ? static_cast<uint32_t>(n) : kWave;
    };
    const auto scales_at = [&](const Pieces<V>& p, int i) {
        return row_of(a.scales, (p.row[i] * a.groups) * 4, units_at(p, i) == 0 ? 0u : static_cast<uint32_t>(a.groups) * 4u);
    };
    const auto fetch = [&](const Pieces<V>& p, Step& q) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int64_t at = p.row[i] * a.units + static_cast<int64_t>(p.col[i]) * kWave;
            const uint32_t n = units_at(p, i);
            if constexpr (BACK) {
                q.code[i] = load_codes(row_of(a.codes, at * 8, n * 8), lane);
                q.s[i] = load_float(scales_at(p, i), ((static_cast<uint32_t>(p.col[i]) * kWave + lane) >> a.lanes_log2) * 4u);
            } else {
                load_unit<Tag>(row_of(a.x, at * Unit<Tag>::kBytes, n * Unit<Tag>::kBytes), lane, q.x[i]);
            }
        }
    };
    const auto advance = [&] {
        r += a.row_step;
        c += a.piece_step;
        if (c >= a.per_row) {
            c -= a.per_row;
            ++r;
        }
    };
    Pieces<V> cur;
    cur.set(r, c, a.per_row);
    Step now;
    fetch(cur, now);
    while (r < a.rows) {
        advance();
        Pieces<V> next;
        next.set(r, c, a.per_row);
        Step then;
        fetch(next, then);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int64_t at = cur.row[i] * a.units + static_cast<int64_t>(cur.col[i]) * kWave;
            const uint32_t n = units_at(cur, i);
            float v[8];
            if constexpr (BACK) {
                decode<C>(now.code[i], v);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= now.s[i];
                u32x4 o[NV];
                Unit<Tag>::pack(v, o);
                store_unit<Tag>(row_of(a.x, at * Unit<Tag>::kBytes, n * Unit<Tag>::kBytes), lane, o);
            } else {
                const Scale sc = scale_of<C>(group_max(Unit<Tag>::amax_bits(now.x[i]), a.lanes_log2));
                Unit<Tag>::unpack(now.x[i], v);
                store_codes(row_of(a.codes, at * 8, n * 8), lane, encode<C>(v, sc), a.keep);
                const uint32_t u = static_cast<uint32_t>(cur.col[i]) * kWave + lane;
                const bool leads = lane < n && (lane & ((1u << a.lanes_log2) - 1u)) == 0;
                store_float(scales_at(cur, i), leads ? (u >> a.lanes_log2) * 4u : kNowhere, sc.s);
            }
        }
        cur = next;
        now = then;
    }
}

}  // namespace lnmod
