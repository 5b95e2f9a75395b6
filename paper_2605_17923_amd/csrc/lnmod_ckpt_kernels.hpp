// lnmod_ckpt_kernels.hpp -- gfx950 device code of LayerNorm-Modulate with an 8-bit checkpoint of x.
//
// The forward writes, beside y and the statistics, the codes of x (lnmod_code.hpp) in the same pass; the backward reads
// them in x's place:
//
//   x'[n,d] = code*s     xhat = (x' - mean_n) * rstd_n     g = dy*(1 + scale)     c1 = mean g     c2 = mean g*xhat
//   dx = rstd_n*(g - c1 - xhat*c2)     dshift = sum_n dy     dscale = sum_n dy*xhat
//
// mean and rstd are those of x itself.  What the two passes save is memory between them, one byte per feature where bf16
// keeps two, and the same byte per feature in the backward's traffic.
//
// The layout is that of the kernels that keep x (lnmod_kernels.hpp): K waves share a row, a lane owns fixed features, so
// the modulation and the running sums stay in registers; rows stay packed and are unpacked per pass; the next step's rows
// are requested before the current step is computed.  Here a lane's unit is eight features in either element type, so that
// a group of codes is 4, 8 or 16 neighbouring lanes and its scale needs no LDS.
//
// Both passes are bound by HBM; their arithmetic (19 to 28 vector operations per feature forward, 15 to 19 backward) keeps the SIMDs
// issuing for half of the time and more, and has to hide behind the loads.  Measured, int8, groups of 128, bytes that have to move:
//   75 600 x 5120 bf16   forward 337 us, 5.8 TB/s    backward 312 us, 6.2 TB/s (+ 5 us second pass)
//   32 760 x 1536 bf16   forward 45 us, 5.6 TB/s     backward 44 us, 5.8 TB/s (+ 4 us)
//   modulation per token, 32 760 x 5120 bf16: forward 252 us, 6.0 TB/s, backward 328 us, 5.6 TB/s
// (a copy reaches 6.1 TB/s).  Three or four steps in registers in place of two, and waves with neighbouring chunks in place of
// chunks K*64 apart, brought nothing.
#pragma once
#include "lnmod_code.hpp"

namespace lnmod {

struct Codes {
    void* codes;             // [N, D] bytes
    float* scales;           // [N, groups]
    int32_t groups;
    int32_t lanes_log2;      // of a group
    int32_t keep;            // forward: codes stored for a reader soon (see keep_codes)
};

struct CkptFwdArgs {
    FwdArgs f;               // nchunks: units of a row
    Codes c;
};

struct CkptBwdArgs {
    BwdArgs b;               // x is not read
    Codes c;
};

constexpr int waves_for(int regs, int most = LNMOD_MAX_WAVES_PER_EU) {
    const int w = 512 / regs;
    return w > most ? most : w < 1 ? 1 : w;
}
constexpr int ckpt_fwd_waves(int vpl, int nv, int r, bool tok) {
    return waves_for(vpl * ((tok ? 0 : 16) + kDepth * r * 4 * nv * (tok ? 3 : 1)) + 56);
}
constexpr int ckpt_bwd_waves(int vpl, int nv, int r, bool tok) {
    return waves_for(vpl * ((tok ? 16 : 24) + kDepth * r * (4 * nv * (tok ? 2 : 1) + 3)) + 56);
}

template <typename Tag, typename C, int VPL, int K, int R, bool TOK>
__global__ __launch_bounds__(K* kWave* fwd_groups_most(K))
LNMOD_OCCUPANCY(ckpt_fwd_waves(VPL, Unit<Tag>::NV, R, TOK))
void ckpt_fwd_kernel(const CkptFwdArgs args) {
    using U = Unit<Tag>;
    constexpr int NV = U::NV, NS = TOK ? 3 : 1;              // streamed inputs per row: x (, scale, shift)
    const FwdArgs& a = args.f;
    const Codes& cd = args.c;
    __shared__ float part[2][R][K][2];

    const int lane = threadIdx.x & (kWave - 1);
    const int in_block = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave = K > 1 ? in_block : 0;   // of the row
    const int groups = K > 1 ? 1 : static_cast<int>(blockDim.x) >> 6, group = K > 1 ? 0 : in_block;
    const int64_t row_bytes = static_cast<int64_t>(a.D) * IO<Tag>::kBytes;

    uint32_t chunk[VPL], scale_off[VPL];                     // scale_off: the group's first lane stores its scale
    bool ok[VPL];
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        chunk[i] = static_cast<uint32_t>((i * K + wave) * kWave + lane);
        ok[i] = chunk[i] < static_cast<uint32_t>(a.nchunks);
        scale_off[i] = ok[i] && (lane & ((1 << cd.lanes_log2) - 1)) == 0 ? (chunk[i] >> cd.lanes_log2) * 4u : kNowhere;
    }
    const uint32_t first_lane = lane == 0 && wave == 0 ? 0u : kNowhere;
    float cnt[K], my_cnt = 0.0f;                             // features each wave holds
#pragma unroll
    for (int w = 0; w < K; ++w) {
        int n = 0;
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            int left = a.nchunks - (i * K + w) * kWave;
            left = left < 0 ? 0 : left > kWave ? kWave : left;
            n += left;
        }
        cnt[w] = static_cast<float>(n * kUnit);
        my_cnt = wave == w ? cnt[w] : my_cnt;
    }
    const float inv_my_cnt = my_cnt > 0.0f ? 1.0f / my_cnt : 0.0f;

    const Place at = place_of(a.split, a.interleave);
    const int64_t r0 = at.cluster * a.rows_per_cluster;
    int64_t stop = r0 + a.rows_per_cluster;
    if (stop > a.T) stop = a.T;
    const int64_t first = r0 + (at.member * groups + group) * R, step = static_cast<int64_t>(a.nb) * groups * R;

    const uint32_t unit_bytes = static_cast<uint32_t>(row_bytes);

    // the modulation row of segment m lives in registers until a row of another segment comes; seg_end is where m's rows end
    float A[TOK ? 1 : VPL][8], B[TOK ? 1 : VPL][8];
    int64_t m = 0, seg_end = a.T;
    const auto load_modulation = [&] {
        const Row rsc = row_of(a.scale, m * row_bytes, unit_bytes), rsh = row_of(a.shift, m * row_bytes, unit_bytes);
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            u32x4 sc[NV], sh[NV];
            load_unit<Tag, 0>(rsc, chunk[i], sc);
            load_unit<Tag, 0>(rsh, chunk[i], sh);
            U::unpack(sc, A[i]);
            U::unpack(sh, B[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) A[i][e] += 1.0f;
        }
    };
    const auto fetch = [&](int64_t base, u32x4 (&q)[NS][R][VPL][NV]) {
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int64_t row = base + j;
            const uint32_t bytes = row < stop ? unit_bytes : 0u;
            const Row rx = row_of(a.x, row * row_bytes, bytes);
#pragma unroll
            for (int i = 0; i < VPL; ++i) load_unit<Tag>(rx, chunk[i], q[0][j][i]);
            if constexpr (TOK) {
                const Row rsc = row_of(a.scale, row * row_bytes, bytes), rsh = row_of(a.shift, row * row_bytes, bytes);
#pragma unroll
                for (int i = 0; i < VPL; ++i) {
                    load_unit<Tag>(rsc, chunk[i], q[NS - 2][j][i]);
                    load_unit<Tag>(rsh, chunk[i], q[NS - 1][j][i]);
                }
            }
        }
    };
    u32x4 bufs[kDepth][NS][R][VPL][NV];
#pragma unroll
    for (int d = 0; d < kDepth - 1; ++d) fetch(first + d * step, bufs[d]);
    if constexpr (!TOK) {
        m = find_segment(a.seg, first < stop ? first : r0);
        if (a.seg.nseg > 1) seg_end = m + 1 < a.seg.nseg ? seg_begin(a.seg, m + 1) : a.T;
        load_modulation();
    }

    int buf = 0;
    const auto compute = [&](int64_t base, u32x4 (&raw)[NS][R][VPL][NV]) {
        // this wave's part of each row: mean, then centred sum of squares; the parts are merged by
        // M2 = sum_k M2_k + sum_k n_k (mean_k - mean)^2
        float mu[R], rs[R];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < VPL; ++i) {
                float v[8];
                U::unpack(raw[0][j][i], v);
#pragma unroll
                for (int e = 0; e < 8; ++e) s += v[e];
            }
            mu[j] = wave_sum(s) * inv_my_cnt;
            float q2 = 0.0f;
#pragma unroll
            for (int i = 0; i < VPL; ++i) {
                float v[8], t = 0.0f;
                U::unpack(raw[0][j][i], v);
#pragma unroll
                for (int e = 0; e < 8; ++e) t += (v[e] - mu[j]) * (v[e] - mu[j]);
                q2 += ok[i] ? t : 0.0f;
            }
            rs[j] = wave_sum(q2);
        }
        if constexpr (K > 1) {
            if (lane == 0) {
#pragma unroll
                for (int j = 0; j < R; ++j) {
                    part[buf][j][wave][0] = mu[j];
                    part[buf][j][wave][1] = rs[j];
                }
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < R; ++j) {
                float sum = 0.0f;
#pragma unroll
                for (int w = 0; w < K; ++w) sum += cnt[w] * part[buf][j][w][0];
                const float mean = sum * a.inv_D;
                float m2 = 0.0f;
#pragma unroll
                for (int w = 0; w < K; ++w) {
                    const float d = part[buf][j][w][0] - mean;
                    m2 += part[buf][j][w][1] + cnt[w] * d * d;
                }
                mu[j] = mean;
                rs[j] = m2;
            }
            buf ^= 1;
        }
#pragma unroll
        for (int j = 0; j < R; ++j) {
            rs[j] = rsqrtf(rs[j] * a.inv_D + a.eps);
#pragma unroll
            for (int i = 0; i < VPL; ++i) opaque(raw[0][j][i]);
        }
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int64_t row = base + j;
            if (row < stop) {
                if (!TOK && row >= seg_end) {
                    // the walk stays inside the table whatever the table holds
                    while (m + 1 < a.seg.nseg && seg_begin(a.seg, m + 1) <= row) ++m;
                    seg_end = m + 1 < a.seg.nseg ? seg_begin(a.seg, m + 1) : a.T;
                    if (seg_end <= row) seg_end = row + 1;
                    load_modulation();
                }
                store_float(row_of(a.mean, row * 4, 4), first_lane, mu[j]);
                store_float(row_of(a.rstd, row * 4, 4), first_lane, rs[j]);
                const Row ry = row_of(a.y, row * row_bytes, unit_bytes), rc = row_of(cd.codes, row * a.D, static_cast<uint32_t>(a.D));
                const Row rcs = row_of(cd.scales, row * cd.groups * 4, static_cast<uint32_t>(cd.groups) * 4u);
#pragma unroll
                for (int i = 0; i < VPL; ++i) {
                    // lanes beyond the row hold zeros
                    const Scale sc = scale_of<C>(group_max(U::amax_bits(raw[0][j][i]), cd.lanes_log2));
                    float v[8], o[8];
                    U::unpack(raw[0][j][i], v);
                    store_codes(rc, chunk[i], encode<C>(v, sc), cd.keep);
                    store_float(rcs, scale_off[i], sc.s);
                    if constexpr (TOK) {
                        float p[8], t[8];
                        U::unpack(raw[NS - 2][j][i], p);
                        U::unpack(raw[NS - 1][j][i], t);
#pragma unroll
                        for (int e = 0; e < 8; ++e) o[e] = ((v[e] - mu[j]) * rs[j]) * (1.0f + p[e]) + t[e];
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) o[e] = ((v[e] - mu[j]) * rs[j]) * A[i][e] + B[i][e];
                    }
                    u32x4 y[NV];
                    U::pack(o, y);
                    store_unit<Tag>(ry, chunk[i], y);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
    };
    for (int64_t base = first; base < stop;) {
#pragma unroll
        for (int d = 0; d < kDepth; ++d) {
            if (base >= stop) break;
            fetch(base + (kDepth - 1) * step, bufs[(d + kDepth - 1) % kDepth]);
            __builtin_amdgcn_sched_barrier(0);               // keep the requests up here
            compute(base, bufs[d]);
            base += step;
        }
    }
}

// Backward.  xhat is one fused step from the code: xhat = code*p + b with p = s*rstd and b = -mean*rstd per unit.  The
// three roundings leave at most 2^-23 (|x'| + |mean|) rstd, a 2^14-th of half a code's step where the group is not far from the
// row's mean; x' - mean first would spare those and cost two operations more per feature.
template <typename Tag, typename C, int VPL, int K, int R, bool TOK>
__global__ __launch_bounds__(K* kWave* (TOK ? 1 : groups_most(K, ckpt_bwd_waves(VPL, Unit<Tag>::NV, R, TOK))))
LNMOD_OCCUPANCY(ckpt_bwd_waves(VPL, Unit<Tag>::NV, R, TOK))
void ckpt_bwd_kernel(const CkptBwdArgs args) {
    using U = Unit<Tag>;
    constexpr int NV = U::NV;
    const BwdArgs& a = args.b;
    const Codes& cd = args.c;
    __shared__ float part[2][R][K][2];
    extern __shared__ f32x4 sums[];          // see add_groups

    const int lane = threadIdx.x & (kWave - 1);
    const int in_block = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave = K > 1 ? in_block : 0;   // of the row
    const int groups = K > 1 || TOK ? 1 : static_cast<int>(blockDim.x) >> 6, group = K > 1 || TOK ? 0 : in_block;
    const int64_t row_bytes = static_cast<int64_t>(a.D) * IO<Tag>::kBytes;

    const uint32_t unit_bytes = static_cast<uint32_t>(row_bytes);

    uint32_t chunk[VPL], scale_off[VPL];
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        chunk[i] = static_cast<uint32_t>((i * K + wave) * kWave + lane);
        scale_off[i] = (chunk[i] >> cd.lanes_log2) * 4u;
    }
    const Place at = place_of(a.split, a.interleave);
    const int64_t cluster = at.cluster, member = at.member * groups + group;
    const int32_t members = a.nb * groups;
    int64_t r0 = cluster * a.rows_per_cluster;
    int64_t r1 = r0 + a.rows_per_cluster;
    if (r1 > a.T) r1 = a.T;
    int buf = 0;
    uint32_t turn = 0;                       // see take_turn

    struct Rows {
        u32x4 dy[R][VPL][NV], sc[TOK ? R : 1][TOK ? VPL : 1][NV];
        u32x2 code[R][VPL];
        float s[R][VPL], mu[R], rs[R];
    };

    while (r0 < r1) {
        int64_t m = 0, stop = r1;
        if (!TOK) {
            m = find_segment(a.seg, r0);
            stop = seg_begin(a.seg, m + 1);
            if (stop > r1) stop = r1;
            if (stop <= r0) stop = r0 + 1;   // malformed table: still make progress
        }
        const auto fetch = [&](int64_t base, Rows& q) {
#pragma unroll
            for (int j = 0; j < R; ++j) {
                const int64_t row = base + j;
                const bool live = row < stop;
                const uint32_t on = live ? ~0u : 0u;
                const int64_t of = live ? row : stop - 1;    // a row beyond the last: statistics 0, everything else reads as 0
                q.mu[j] = live ? float_at(a.mean, of) : 0.0f;
                q.rs[j] = live ? float_at(a.rstd, of) : 0.0f;
                const Row rdy = row_of(a.dy, row * row_bytes, unit_bytes & on);
                const Row rc = row_of(cd.codes, row * a.D, static_cast<uint32_t>(a.D) & on);
                const Row rcs = row_of(cd.scales, row * cd.groups * 4, (static_cast<uint32_t>(cd.groups) * 4u) & on);
#pragma unroll
                for (int i = 0; i < VPL; ++i) {
                    load_unit<Tag>(rdy, chunk[i], q.dy[j][i]);
                    q.code[j][i] = load_codes(rc, chunk[i]);
                    q.s[j][i] = load_float(rcs, scale_off[i]);
                }
                if constexpr (TOK) {
                    const Row rsc = row_of(a.scale, row * row_bytes, unit_bytes & on);
#pragma unroll
                    for (int i = 0; i < VPL; ++i) load_unit<Tag>(rsc, chunk[i], q.sc[j][i]);
                }
            }
        };
        const int64_t step = static_cast<int64_t>(members) * R;
        const int64_t first = take_turn<R>(turn, r0, stop, member, members);
        Rows bufs[kDepth];
#pragma unroll
        for (int d = 0; d < kDepth - 1; ++d) fetch(first + d * step, bufs[d]);

        float A[TOK ? 1 : VPL][8], acc[2][TOK ? 1 : VPL][8];
        float(&acc_s)[TOK ? 1 : VPL][8] = acc[0], (&acc_c)[TOK ? 1 : VPL][8] = acc[1];
        if constexpr (!TOK) {
            const Row rsc = row_of(a.scale, m * row_bytes, unit_bytes);
#pragma unroll
            for (int i = 0; i < VPL; ++i) {
                u32x4 r[NV];
                load_unit<Tag, 0>(rsc, chunk[i], r);
                U::unpack(r, A[i]);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    A[i][e] += 1.0f;
                    acc_s[i][e] = 0.0f;
                    acc_c[i][e] = 0.0f;
                }
            }
        }

        const auto compute = [&](int64_t base, Rows& now) {
            float c1[R], c2[R];
#pragma unroll
            for (int j = 0; j < R; ++j) {
                float p1 = 0.0f, p2 = 0.0f;
                const float b = -now.mu[j] * now.rs[j];
#pragma unroll
                for (int i = 0; i < VPL; ++i) {
                    float dyv[8], cv[8], scv[8];
                    U::unpack(now.dy[j][i], dyv);
                    decode<C>(now.code[j][i], cv);
                    if constexpr (TOK) U::unpack(now.sc[j][i], scv);
                    const float p = now.s[j][i] * now.rs[j];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float h = __builtin_fmaf(cv[e], p, b);
                        const float g = dyv[e] * (TOK ? 1.0f + scv[e] : A[TOK ? 0 : i][e]);
                        p1 += g;
                        p2 += g * h;                         // lanes beyond the row: dy = 0
                        if constexpr (!TOK) {
                            acc_s[i][e] += dyv[e];
                            acc_c[i][e] += dyv[e] * h;
                        }
                    }
                    if constexpr (!TOK) {
                        // pinned here, or the optimiser sinks these adds below the barrier
#pragma unroll
                        for (int e = 0; e < 8; ++e) asm volatile("" : "+v"(acc_s[i][e]), "+v"(acc_c[i][e]));
                    }
                    __builtin_amdgcn_sched_barrier(0);       // one unit at a time
                }
                c1[j] = wave_sum(p1);
                c2[j] = wave_sum(p2);
            }
            if constexpr (K > 1) {
                if (lane == 0) {
#pragma unroll
                    for (int j = 0; j < R; ++j) {
                        part[buf][j][wave][0] = c1[j];
                        part[buf][j][wave][1] = c2[j];
                    }
                }
                __syncthreads();
#pragma unroll
                for (int j = 0; j < R; ++j) {
                    float t1 = 0.0f, t2 = 0.0f;
#pragma unroll
                    for (int w = 0; w < K; ++w) {
                        t1 += part[buf][j][w][0];
                        t2 += part[buf][j][w][1];
                    }
                    c1[j] = t1;
                    c2[j] = t2;
                }
                buf ^= 1;
            }
#pragma unroll
            for (int j = 0; j < R; ++j) {
#pragma unroll
                for (int i = 0; i < VPL; ++i) {
                    opaque(now.dy[j][i]);
                    asm volatile("" : "+v"(now.code[j][i]));
                }
            }
#pragma unroll
            for (int j = 0; j < R; ++j) {
                const int64_t row = base + j;
                if (row < stop) {
                    const float b = -now.mu[j] * now.rs[j];
                    // rstd*(g - c1 - xhat*c2) with xhat = code*p + b
                    const float k1 = now.rs[j] * (c1[j] * a.inv_D), k2 = now.rs[j] * (c2[j] * a.inv_D);
                    const float bk = -(k1 + b * k2);
                    const Row rdx = row_of(a.dx, row * row_bytes, unit_bytes);
#pragma unroll
                    for (int i = 0; i < VPL; ++i) {
                        float dyv[8], cv[8], scv[8], o[8], ds[8];
                        U::unpack(now.dy[j][i], dyv);
                        decode<C>(now.code[j][i], cv);
                        if constexpr (TOK) U::unpack(now.sc[j][i], scv);
                        const float p = now.s[j][i] * now.rs[j], pk = -p * k2;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float g = dyv[e] * (TOK ? 1.0f + scv[e] : A[TOK ? 0 : i][e]);
                            o[e] = __builtin_fmaf(g, now.rs[j], __builtin_fmaf(cv[e], pk, bk));
                            if constexpr (TOK) ds[e] = dyv[e] * __builtin_fmaf(cv[e], p, b);
                        }
                        u32x4 t[NV];
                        U::pack(o, t);
                        store_unit<Tag>(rdx, chunk[i], t);
                        if constexpr (TOK) {                 // dshift = dy as loaded, dscale = dy*xhat
                            store_unit<Tag>(row_of(a.dshift, row * row_bytes, unit_bytes), chunk[i], now.dy[j][i]);
                            U::pack(ds, t);
                            store_unit<Tag>(row_of(a.dscale, row * row_bytes, unit_bytes), chunk[i], t);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
        };
        for (int64_t base = first; base < stop;) {
#pragma unroll
            for (int d = 0; d < kDepth; ++d) {
                if (base >= stop) break;
                fetch(base + (kDepth - 1) * step, bufs[(d + kDepth - 1) % kDepth]);
                __builtin_amdgcn_sched_barrier(0);           // keep the requests up here
                compute(base, bufs[d]);
                base += step;
            }
        }

        if constexpr (!TOK) {
            // this block's partial sums for segment m (slots: see bwd_seg_kernel)
            add_groups<units_at_once(VPL, ckpt_bwd_waves(VPL, NV, R, TOK))>(acc, group, groups, sums);
            const int64_t slot = ((cluster + m) * a.nb + at.member) * 2 * a.D * 4;
            const uint32_t bytes = group == 0 ? static_cast<uint32_t>(a.D) * 4u : 0u;
            const Row ps = row_of(a.ws, slot, bytes);
            const Row pc = row_of(a.ws, slot + static_cast<int64_t>(a.D) * 4, bytes);
#pragma unroll
            for (int i = 0; i < VPL; ++i) {
                store_sums8(ps, chunk[i], acc_s[i]);
                store_sums8(pc, chunk[i], acc_c[i]);
            }
        }
        r0 = stop;
    }
}

}  // namespace lnmod
