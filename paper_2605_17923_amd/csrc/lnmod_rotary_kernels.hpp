// lnmod_rotary_kernels.hpp -- gfx950 device code of rotary positions with several axes, and of the query and key norm with
// the rotation in the same pass.
//
//   pair j of a head, with the token's position p on the pair's axis and (c, s) = table[p][j]:
//     (u, v) -> (u c - v s, u s + v c)            backwards (c, -s)
//   norm first (the whole token's row, or each head's):  rstd = 1/sqrt(mean x^2 + eps)   x -> (x rstd) w
//   its backward, with g' the gradient turned back:  xhat = x rstd   g = g' w   c = mean g xhat
//     dx = rstd (g - xhat c)   dw = sum over tokens (and heads, if a head has the norm) of g' xhat
//
// A head is split into units of sixteen bytes that hold whole pairs: consecutive features where a pair is two neighbours, two
// runs of eight bytes R/2 features apart where a pair is j and j + R/2.  A lane keeps one unit's place for the whole life of
// its block and meets that place in several heads of a token, so the four (fp32: two) cosines and sines that it needs for a
// token are loaded once for all of them.  Lanes without a unit of their own read a neighbour's and write nothing.
//
// HBM bounds the large ones: 75 600 x 40 x 128 bf16, queries and keys, 533 us, 5.8 TB/s; with the norm over rows 32 760 x 40 x 128
// from dense tensors 243 us forwards (5.5 TB/s), 335 backwards (6.0), 342 with gradients that have the heads in front.  The
// next token's units are loaded while this one's are worked on.
//
// Two forms are further from it.  Pairs of halves are loaded and stored by runs of eight bytes, twice the accesses: the same row
// backward 331 us in pairs, 401 in halves, the rotation alone 225 and 258.  Heads of 96 features leave a quarter of the lanes idle, of 72
// seven of sixteen, as a head's lanes are a power of two: 24 + 8 x 96, a norm for each head, 28 837 tokens 84 us forwards and 105
// backwards in pairs, 95 and 127 in halves, where the bytes ask for 59 and 89.
#pragma once
#include "lnmod_kernels.hpp"
#include "lnmod_rotary.hpp"

namespace lnmod {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Where the features of a lane's unit lie in a head, and the pairs they are.
template <typename Tag, bool HALVES>
struct UnitPlace {
    static constexpr int E = IO<Tag>::E, P = E / 2;
    uint32_t lo, hi;                 // byte offsets of the unit's halves (hi: the second eight bytes)
    int32_t pair;                    // the first pair
    bool turned[P];
    int32_t axis[P];

    __device__ inline UnitPlace(const RotaryPlan& r, int u) {
        pair = u * P;
        bool whole = true;           // HALVES: a unit of turned features
        if (HALVES) whole = u * P < r.half;
        const int first = HALVES && whole ? u * P : u * E;
        lo = static_cast<uint32_t>(first) * IO<Tag>::kBytes;
        hi = HALVES && whole ? lo + static_cast<uint32_t>(r.half) * IO<Tag>::kBytes : lo + 8u;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int j = pair + i;
            turned[i] = j < r.half;
            int a = 0;
#pragma unroll
            for (int k = 1; k < kMaxAxes; ++k) a += j >= r.first[k] ? 1 : 0;
            axis[i] = a < r.axes ? a : 0;
        }
    }
    // value e of the unit -> the pair it belongs to, and its place in the pair
    __device__ static constexpr int pair_of(int e) { return HALVES ? e % P : e / 2; }
    __device__ static constexpr int first_of(int i) { return HALVES ? i : 2 * i; }
    __device__ static constexpr int second_of(int i) { return HALVES ? i + P : 2 * i + 1; }
    // feature of value e
    __device__ inline int feature(int e) const {
        return static_cast<int>((e < P ? lo : hi) / IO<Tag>::kBytes) + (e < P ? e : e - P);
    }

    // Runs of eight bytes share their lines with another access of the wave, which finds them in the cache (24 x 96 bf16, a norm
    // for each head, 130 us past the caches, 120 so).
    __device__ inline u32x4 load(const char* head) const {
        if (!HALVES) return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(head + lo));
        return load_cached(head);
    }
    __device__ inline u32x4 load_cached(const char* head) const {
        if (!HALVES) return *reinterpret_cast<const u32x4*>(head + lo);
        const u32x2 a = *reinterpret_cast<const u32x2*>(head + lo), b = *reinterpret_cast<const u32x2*>(head + hi);
        return u32x4{a[0], a[1], b[0], b[1]};
    }
    __device__ inline void store(char* head, const u32x4& v) const {
        if (!HALVES) {
            __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(head + lo));
            return;
        }
        *reinterpret_cast<u32x2*>(head + lo) = u32x2{v[0], v[1]};
        *reinterpret_cast<u32x2*>(head + hi) = u32x2{v[2], v[3]};
    }
};

template <int P> struct Angles {
    float c[P], s[P];
};

// A token's positions on the axes of a lane's pairs.
template <typename Tag, bool HALVES>
__device__ inline void positions_of(const RotaryPlan& r, const UnitPlace<Tag, HALVES>& at, int64_t row, int32_t (&p)[IO<Tag>::E / 2]) {
    const int32_t* pos = r.positions + row * r.axes;
#pragma unroll
    for (int i = 0; i < IO<Tag>::E / 2; ++i) p[i] = pos[at.axis[i]];
}

// The cosines and sines of the pairs there.  A position outside the table has none: NaN.
template <typename Tag, bool HALVES>
__device__ inline void angles_of(const RotaryPlan& r, const UnitPlace<Tag, HALVES>& at, const int32_t (&pos)[IO<Tag>::E / 2],
                                 Angles<IO<Tag>::E / 2>& out) {
#pragma unroll
    for (int i = 0; i < IO<Tag>::E / 2; ++i) {
        const uint32_t p = static_cast<uint32_t>(pos[i]);
        const bool known = p < r.table_rows;
        const int64_t e = static_cast<int64_t>(known ? p : 0u) * r.half + (at.turned[i] ? at.pair + i : 0);
        const f32x2 t = *reinterpret_cast<const f32x2*>(r.table + 2 * e);
        out.c[i] = known ? t[0] : __builtin_nanf("");
        out.s[i] = known ? t[1] : __builtin_nanf("");
    }
}

// Features beyond the turned ones pass as they are, whatever stands in them.
template <typename Tag, bool HALVES>
__device__ inline void turn(const RotaryPlan& r, const UnitPlace<Tag, HALVES>& at, const Angles<IO<Tag>::E / 2>& t, float sign,
                            float (&v)[IO<Tag>::E]) {
#pragma unroll
    for (int i = 0; i < IO<Tag>::E / 2; ++i) {
        const int a = at.first_of(i), b = at.second_of(i);
        const float u = v[a], w = v[b], s = t.s[i] * sign;
        const float x = __builtin_fmaf(u, t.c[i], -(w * s)), y = __builtin_fmaf(u, s, w * t.c[i]);
        v[a] = !r.part || at.turned[i] ? x : u;
        v[b] = !r.part || at.turned[i] ? y : w;
    }
}

// Sum over the 2^bits neighbouring lanes that a lane is one of (bits uniform); every one of them returns it.
__device__ inline float lanes_sum(float v, int bits) {
    if (bits == 6) return wave_sum(v);
    const auto step = [](float x, float t, bool on) { return on ? x + t : x; };
    const auto dpp = [](float x, auto ctrl) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xf, 0xf, false));
    };
    v = step(v, dpp(v, std::integral_constant<int, 0xB1>{}), bits > 0);
    v = step(v, dpp(v, std::integral_constant<int, 0x4E>{}), bits > 1);
    v = step(v, dpp(v, std::integral_constant<int, 0x141>{}), bits > 2);
    v = step(v, dpp(v, std::integral_constant<int, 0x140>{}), bits > 3);
    if (bits > 4) v += __shfl_xor(v, 16);
    return v;
}

// What a wave works on: a token's heads are shared out over the waves of a team and, inside a wave, over 2^hs_log2 groups of
// 2^g_log2 lanes; a token with fewer heads than a wave has groups leaves room for its neighbours in the same wave.
struct Lanes {
    int lane, wave, u, slot, sub, team, part;
    bool unit, live;
    __device__ inline Lanes(const RotaryArgs& a, int t) {
        lane = threadIdx.x & (kWave - 1);
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int group = lane >> a.g_log2;
        u = lane & ((1 << a.g_log2) - 1);
        unit = u < a.units;
        if (!unit) u = a.units - 1;
        slot = group & ((1 << a.side[t].hs_log2) - 1);
        sub = group >> a.side[t].hs_log2;
        team = wave / a.side[t].waves;
        part = wave - team * a.side[t].waves;
        live = team < a.side[t].teams;
        if (!live) team = part = 0;
    }
};

__device__ inline void zero_unless(bool keep, u32x4& q) {
    const uint32_t m = keep ? ~0u : 0u;
    q &= u32x4{m, m, m, m};
}

// NORM: 0 none, 1 over a token's row, 2 over each head
template <typename Tag, int NORM, bool HALVES, int VPL>
__global__ __launch_bounds__(8 * kWave) LNMOD_OCCUPANCY(VPL <= 3 ? 4 : VPL == 4 ? 3 : 2) void rotary_fwd_kernel(const RotaryArgs a) {
    using io = IO<Tag>;
    constexpr int E = io::E;
    __shared__ float sums[2][8];
    const int t = blockIdx.x >= static_cast<unsigned>(a.side[0].blocks) ? 1 : 0;
    const RotarySide& side = a.side[t];
    const int index = static_cast<int>(blockIdx.x) - (t ? a.side[0].blocks : 0);
    const int64_t member = index / side.chunks;
    const int head0 = (index - static_cast<int>(member) * side.chunks) * side.chunk_heads;
    const Lanes me(a, t);
    const UnitPlace<Tag, HALVES> at(a.rot, me.u);
    const int tokens_log2 = 6 - a.g_log2 - side.hs_log2;             // of a wave

    int64_t in[VPL];
    uint32_t out[VPL];
    bool ok[VPL];
    float W[VPL][E];
    const uint32_t head_bytes = static_cast<uint32_t>(a.head_dim) * io::kBytes;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const int h = head0 + ((i * side.waves + me.part) << side.hs_log2) + me.slot;
        ok[i] = me.unit && me.live && h < side.heads;
        const int hc = h < side.heads ? h : side.heads - 1;
        in[i] = hc * side.x.head;
        out[i] = static_cast<uint32_t>(hc) * head_bytes;
        if (NORM && (NORM == 1 || i == 0))
            io::unpack(at.load_cached(static_cast<const char*>(side.w) + (NORM == 1 ? out[i] : 0u)), W[i]);
    }

    const int64_t stride = (static_cast<int64_t>(side.members) * side.teams) << tokens_log2;
    const int64_t first = ((member * side.teams) << tokens_log2);
    // Positions are loaded two steps ahead where there is no norm, so that a step's angles, which they choose, come with its units
    // and six waves keep a CU's share of HBM busy: 32 760 x 40 x 128 from tensors with the heads in front 248 -> 231 us.  A norm
    // over rows, which waits between its loads and its stores in any case, had nothing of it and paid the longer start
    // (32 760 x 12 x 128 77 -> 85 us).
    constexpr bool kAhead = NORM == 0;
    auto token = [&](int64_t base) {
        const int64_t n = base + (static_cast<int64_t>(me.team) << tokens_log2) + me.sub;
        return n < a.N ? n : a.N - 1;
    };
    int32_t pos[E / 2];
    auto positions = [&](int64_t base) {
        const int64_t n = token(base);
        const uint32_t b = a.rot.per_token ? 0u : a.sample_of(static_cast<uint32_t>(n));
        positions_of(a.rot, at, n - static_cast<int64_t>(b) * a.S, pos);
    };
    auto fetch = [&](int64_t base, u32x4 (&raw)[VPL], Angles<E / 2>& ang) {
        const int64_t n = token(base);
        const uint32_t b = a.sample_of(static_cast<uint32_t>(n)), s = static_cast<uint32_t>(n) - b * a.S;
        const char* x = side.x.p + b * side.x.batch + s * side.x.token;
#pragma unroll
        for (int i = 0; i < VPL; ++i) raw[i] = at.load(x + in[i]);
        if (!kAhead) positions_of(a.rot, at, a.rot.per_token ? n : static_cast<int64_t>(s), pos);
        angles_of(a.rot, at, pos, ang);
    };

    u32x4 raw[VPL];
    Angles<E / 2> ang;
    if (kAhead) positions(first);
    fetch(first, raw, ang);
    if (kAhead) positions(first + stride);
    int buf = 0;
    for (int64_t base = first; base < a.N; base += stride) {
        u32x4 nxt[VPL];
        Angles<E / 2> nang;
        fetch(base + stride, nxt, nang);
        if (kAhead) positions(base + 2 * stride);
        const int64_t n = base + (static_cast<int64_t>(me.team) << tokens_log2) + me.sub;
        const bool here = n < a.N;
        float rs = 1.0f;
        if (NORM == 1) {
            float q = 0.0f;
#pragma unroll
            for (int i = 0; i < VPL; ++i) {
                zero_unless(ok[i], raw[i]);
                float v[E];
                io::unpack(raw[i], v);
#pragma unroll
                for (int e = 0; e < E; ++e) q = __builtin_fmaf(v[e], v[e], q);
            }
            q = lanes_sum(q, a.g_log2 + side.hs_log2);
            if (side.waves > 1) {
                if (me.lane == 0) sums[buf][me.wave] = q;
                __syncthreads();
                q = 0.0f;
                for (int w = 0; w < side.waves; ++w) q += sums[buf][me.team * side.waves + w];
                buf ^= 1;
            }
            rs = 1.0f / sqrtf(q * side.inv_width + a.eps);
            if (here && ok[0] && me.part == 0 && me.slot == 0 && (me.lane & ((1 << a.g_log2) - 1)) == 0) side.rstd[n] = rs;
        }
        char* y = static_cast<char*>(side.y) + n * (static_cast<int64_t>(side.heads) * head_bytes);
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            if (NORM == 2) zero_unless(me.unit, raw[i]);
            float v[E];
            io::unpack(raw[i], v);
            if (NORM == 2) {
                float q = 0.0f;
#pragma unroll
                for (int e = 0; e < E; ++e) q = __builtin_fmaf(v[e], v[e], q);
                q = lanes_sum(q, a.g_log2);
                rs = 1.0f / sqrtf(q * side.inv_width + a.eps);
                if (here && ok[i] && (me.lane & ((1 << a.g_log2) - 1)) == 0)
                    side.rstd[n * side.heads + head0 + ((i * side.waves + me.part) << side.hs_log2) + me.slot] = rs;
            }
            if (NORM) {
#pragma unroll
                for (int e = 0; e < E; ++e) v[e] = (v[e] * rs) * W[NORM == 1 ? i : 0][e];
            }
            turn(a.rot, at, ang, a.sign, v);
            if (here && ok[i]) at.store(y + out[i], io::pack(v));
        }
#pragma unroll
        for (int i = 0; i < VPL; ++i) raw[i] = nxt[i];
        ang = nang;
    }
}

template <typename Tag, int NORM, bool HALVES, int VPL>
__global__ __launch_bounds__(8 * kWave) void rotary_bwd_kernel(const RotaryArgs a) {
    using io = IO<Tag>;
    constexpr int E = io::E;
    constexpr int A = NORM == 1 ? VPL : 1;
    __shared__ float sums[2][8];
    extern __shared__ float shared_dw[];
    const int t = blockIdx.x >= static_cast<unsigned>(a.side[0].blocks) ? 1 : 0;
    const RotarySide& side = a.side[t];
    const int index = static_cast<int>(blockIdx.x) - (t ? a.side[0].blocks : 0);
    const int64_t member = index / side.chunks;
    const int head0 = (index - static_cast<int>(member) * side.chunks) * side.chunk_heads;
    const Lanes me(a, t);
    const UnitPlace<Tag, HALVES> at(a.rot, me.u);
    const int tokens_log2 = 6 - a.g_log2 - side.hs_log2;

    int64_t in[VPL], gin[VPL];
    uint32_t out[VPL];
    bool ok[VPL];
    float W[A][E], acc[A][E];
    const uint32_t head_bytes = static_cast<uint32_t>(a.head_dim) * io::kBytes;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const int h = head0 + ((i * side.waves + me.part) << side.hs_log2) + me.slot;
        ok[i] = me.unit && me.live && h < side.heads;
        const int hc = h < side.heads ? h : side.heads - 1;
        in[i] = hc * side.x.head;
        gin[i] = hc * side.dy.head;
        out[i] = static_cast<uint32_t>(hc) * head_bytes;
        if (i < A) {
            io::unpack(at.load_cached(static_cast<const char*>(side.w) + (NORM == 1 ? out[i] : 0u)), W[i]);
#pragma unroll
            for (int e = 0; e < E; ++e) acc[i][e] = 0.0f;
        }
    }

    const int64_t stride = (static_cast<int64_t>(side.members) * side.teams) << tokens_log2;
    const int64_t first = ((member * side.teams) << tokens_log2);
    // Positions two steps ahead, as forwards without a norm.  32 760 x 40 x 128, a norm over rows, in the best shape of each: 365 us
    // with the positions loaded beside the units, 334 so (gradients with the heads in front 394 and 341).
    auto token = [&](int64_t base) {
        const int64_t n = base + (static_cast<int64_t>(me.team) << tokens_log2) + me.sub;
        return n < a.N ? n : a.N - 1;
    };
    int32_t pos[E / 2];
    auto positions = [&](int64_t base) {
        const int64_t n = token(base);
        const uint32_t b = a.rot.per_token ? 0u : a.sample_of(static_cast<uint32_t>(n));
        positions_of(a.rot, at, n - static_cast<int64_t>(b) * a.S, pos);
    };
    auto fetch = [&](int64_t base, u32x4 (&raw)[VPL], u32x4 (&grad)[VPL], float (&rs)[NORM == 1 ? 1 : VPL], Angles<E / 2>& ang) {
        const int64_t n = token(base);
        const uint32_t b = a.sample_of(static_cast<uint32_t>(n)), s = static_cast<uint32_t>(n) - b * a.S;
        const char* x = side.x.p + b * side.x.batch + s * side.x.token;
        const char* g = side.dy.p + b * side.dy.batch + s * side.dy.token;
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            raw[i] = at.load(x + in[i]);
            grad[i] = at.load(g + gin[i]);
        }
        if (NORM == 1) rs[0] = side.rstd[n];
        else {
#pragma unroll
            for (int i = 0; i < VPL; ++i) {
                const int h = head0 + ((i * side.waves + me.part) << side.hs_log2) + me.slot;
                rs[i] = side.rstd[n * side.heads + (h < side.heads ? h : side.heads - 1)];
            }
        }
        angles_of(a.rot, at, pos, ang);
    };

    u32x4 raw[VPL], grad[VPL];
    float rs[NORM == 1 ? 1 : VPL];
    Angles<E / 2> ang;
    positions(first);
    fetch(first, raw, grad, rs, ang);
    positions(first + stride);
    int buf = 0;
    for (int64_t base = first; base < a.N; base += stride) {
        u32x4 nxt[VPL], ngrad[VPL];
        float nrs[NORM == 1 ? 1 : VPL];
        Angles<E / 2> nang;
        fetch(base + stride, nxt, ngrad, nrs, nang);
        positions(base + 2 * stride);
        const int64_t n = base + (static_cast<int64_t>(me.team) << tokens_log2) + me.sub;
        const bool here = n < a.N;
        // gradients that do not count are zeros: x beside them is a row's own, so that no product is NaN but the row's own
#pragma unroll
        for (int i = 0; i < VPL; ++i) zero_unless(here && ok[i], grad[i]);
        float c = 0.0f;
        if (NORM == 1) {
#pragma unroll
            for (int i = 0; i < VPL; ++i) {
                float x[E], g[E];
                io::unpack(raw[i], x);
                io::unpack(grad[i], g);
                turn(a.rot, at, ang, -1.0f, g);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float p = g[e] * (x[e] * rs[0]);
                    c = __builtin_fmaf(p, W[i][e], c);
                    acc[i][e] += p;
                }
            }
            c = lanes_sum(c, a.g_log2 + side.hs_log2);
            if (side.waves > 1) {
                if (me.lane == 0) sums[buf][me.wave] = c;
                __syncthreads();
                c = 0.0f;
                for (int w = 0; w < side.waves; ++w) c += sums[buf][me.team * side.waves + w];
                buf ^= 1;
            }
        }
        char* dx = static_cast<char*>(side.y) + n * (static_cast<int64_t>(side.heads) * head_bytes);
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            float x[E], g[E];
            io::unpack(raw[i], x);
            io::unpack(grad[i], g);
            turn(a.rot, at, ang, -1.0f, g);
            const float r = rs[NORM == 1 ? 0 : i];
            if (NORM == 2) {
                c = 0.0f;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float p = g[e] * (x[e] * r);
                    c = __builtin_fmaf(p, W[0][e], c);
                    acc[0][e] += p;
                }
                c = lanes_sum(c, a.g_log2);
            }
            const float k = c * side.inv_width;
#pragma unroll
            for (int e = 0; e < E; ++e) g[e] = r * (g[e] * W[NORM == 1 ? i : 0][e] - (x[e] * r) * k);
            if (here && ok[i]) at.store(dx + out[i], io::pack(g));
        }
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            raw[i] = nxt[i];
            grad[i] = ngrad[i];
        }
#pragma unroll
        for (int i = 0; i < (NORM == 1 ? 1 : VPL); ++i) rs[i] = nrs[i];
        ang = nang;
    }

    // this block's partial dw: the tokens that a wave holds side by side, then the teams in their order
    float* slot = side.ws + static_cast<int64_t>(index) * side.width;
    const int from = a.g_log2 + (NORM == 1 ? side.hs_log2 : 0);
#pragma unroll
    for (int i = 0; i < A; ++i) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            for (int bit = from; bit < 6; ++bit) acc[i][e] += __shfl_xor(acc[i][e], 1 << bit);
        }
    }
    const int turns = NORM == 1 ? side.teams : side.teams * side.waves;
    const int mine = !me.live ? -1 : NORM == 1 ? me.team : me.wave;
    const bool writes = me.unit && (NORM == 1 ? me.sub == 0 : (me.lane >> a.g_log2) == 0);
    for (int w = 0; w < turns; ++w) {
        if (w == mine && writes) {
#pragma unroll
            for (int i = 0; i < A; ++i) {
                if (NORM == 1 && !ok[i]) continue;
                const uint32_t head = NORM == 1 ? out[i] / io::kBytes : 0u;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const uint32_t f = head + at.feature(e);
                    const float v = w ? shared_dw[f] + acc[i][e] : acc[i][e];
                    if (w == turns - 1) slot[f] = v;
                    else shared_dw[f] = v;
                }
            }
        }
        if (turns > 1) __syncthreads();
    }
}

// Second pass: the slots of both tensors, in an order that only their number sets.  Few bytes that a chain of loads would
// wait for, so a block takes 16 features by 64 slots at a time, eight of those loads under way: 512 slots of 5120 features 6.4 us
// with 64 features by 16 slots, 5.6 us so; 1536 slots of 96 features 4.7 us so.
constexpr int kDwFeatures = 16, kDwRows = 16 * kWave / kDwFeatures;

template <typename Tag>
__global__ __launch_bounds__(16 * kWave) void rotary_dw_kernel(const RotaryDwArgs a) {
    __shared__ float part[kDwRows][kDwFeatures + 1];
    const int at = threadIdx.x % kDwFeatures, row = threadIdx.x / kDwFeatures;
    const int t = blockIdx.y;
    const int f = blockIdx.x * kDwFeatures + at;
    const int width = a.width[t];
    float s = 0.0f;
    if (f < width) {
        const float* from = a.ws[t] + f;
        int i = row;
        for (; i + 7 * kDwRows < a.slots[t]; i += 8 * kDwRows) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = from[static_cast<int64_t>(i + j * kDwRows) * width];
#pragma unroll
            for (int j = 0; j < 8; ++j) s += v[j];
        }
        float v[7];                                                  // fewer than eight are left
#pragma unroll
        for (int j = 0; j < 7; ++j) {
            const int slot = i + j * kDwRows;
            v[j] = slot < a.slots[t] ? from[static_cast<int64_t>(slot) * width] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 7; ++j) s += v[j];
    }
    part[row][at] = s;
    __syncthreads();
    if (row >= 4 || f >= width) return;                              // one wave; its four rows add sixteen each
    s = 0.0f;
#pragma unroll
    for (int j = 0; j < kDwRows / 4; ++j) s += part[row * (kDwRows / 4) + j][at];
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    if (row) return;
    if constexpr (std::is_same<Tag, bf16_io>::value) static_cast<__bf16*>(a.dw[t])[f] = static_cast<__bf16>(s);
    else static_cast<float*>(a.dw[t])[f] = s;
}

}  // namespace lnmod
