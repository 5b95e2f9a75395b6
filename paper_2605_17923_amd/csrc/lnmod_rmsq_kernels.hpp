// lnmod_rmsq_kernels.hpp -- gfx950 device code of the root-mean-square norm with the residual's addition and an output in
// 8 bits.
//
//   h = x + r, one fp32 addition rounded once to the I/O type and stored (without a residual h is x, and not stored)
//   rstd_n = 1/sqrt(mean_d h^2 + eps)      v = (h*rstd_n)*w
//   out: the codes of v and their scales (lnmod_code.hpp), or in the I/O type the values that the codes stand for
//
// Backward, straight through the rounding to codes:
//
//   hhat = h*rstd   g = dy*w   c_n = mean_d g*hhat   dx = dh + rstd*(g - hhat*c)   dw[d] = sum_n dy*hhat
//
// With a scale for the whole row, its largest |v| is rstd times the largest |h*w|, so one barrier carries both the sum of
// squares and the maximum; the maximum then differs from the largest |v| by two roundings at most, and a code whose v*r comes
// out at Q (1 + 2^-21) still rounds to Q.  (eps >= 1e-20 keeps 16 bits of an |h*w| whose v is above the floor of 2^-100; the
// maximum of v itself in a second pass, for rows whose |h*w| leaves the normal numbers, cost registers that every row
// pays for.)  A group's maximum is that of v itself, as it is coded.  Layout and pipeline are those
// of lnmod_ckpt_kernels.hpp.
//
// Bound by HBM (17.4 vector operations per feature forward).  Measured, bf16 with a residual:
//   32 760 x 5120, codes, a scale for a row     forward 198 us, 5.9 TB/s
//   32 760 x 1536, values, groups of 128        forward 65 us, 6.2 TB/s     backward 72 us, 5.6 TB/s (+ 5 us second pass),
//       with the residual's gradient in memory of its own 83 us, 6.1 TB/s
//   1 x 5120 2.4 us, 96 x 4096 3.2 us: a launch and one pass through the memory's latency
#pragma once
#include "lnmod_code.hpp"

namespace lnmod {

struct RmsqFwdArgs {
    const void* x;
    const void* r;
    const void* w;
    void* h;                 // written if there is a residual
    void* out;               // codes or values
    float* scales;           // with codes
    float* rstd;
    int64_t N;
    int32_t nb;              // blocks
    int32_t D;
    int32_t nchunks;         // units of a row
    int32_t groups;          // of a row
    int32_t lanes_log2;      // of a group; 0: the row is one
    int32_t keep;            // see keep_codes
    float eps;
    float inv_D;
};

constexpr int rmsq_waves(int regs) {
    const int w = 512 / regs;
    return w > 4 ? 4 : w < 1 ? 1 : w;
}

// ROW: one scale for a row.  VALUES: out holds the values that the codes stand for.
template <typename Tag, typename C, int VPL, int K, int R, bool RES, bool ROW, bool VALUES>
__global__ __launch_bounds__(K* kWave* fwd_groups_most(K))
LNMOD_OCCUPANCY(rmsq_waves(VPL * (8 + kDepth * R * 4 * Unit<Tag>::NV * (RES ? 2 : 1)) + 48))
void rmsq_fwd_kernel(const RmsqFwdArgs a) {
    using U = Unit<Tag>;
    constexpr int NV = U::NV;
    __shared__ float part[2][R][K][2];
    const int lane = threadIdx.x & (kWave - 1);
    const int in_block = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave = K > 1 ? in_block : 0;   // of the row
    const int groups = K > 1 ? 1 : static_cast<int>(blockDim.x) >> 6, group = K > 1 ? 0 : in_block;
    const int64_t row_bytes = static_cast<int64_t>(a.D) * IO<Tag>::kBytes;
    const uint32_t unit_bytes = static_cast<uint32_t>(row_bytes);

    uint32_t chunk[VPL], scale_off[VPL];                     // scale_off: the group's first lane stores its scale
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        chunk[i] = static_cast<uint32_t>((i * K + wave) * kWave + lane);
        scale_off[i] = chunk[i] < static_cast<uint32_t>(a.nchunks) && (lane & ((1 << a.lanes_log2) - 1)) == 0
                           ? (chunk[i] >> a.lanes_log2) * 4u : kNowhere;
    }
    const uint32_t first_lane = lane == 0 && wave == 0 ? 0u : kNowhere;
    float W[VPL][8];
    struct Rows {
        u32x4 x[R][VPL][NV], r[RES ? R : 1][RES ? VPL : 1][NV];
    };
    const auto fetch = [&](int64_t base, Rows& q) {
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int64_t row = base + j;
            const uint32_t bytes = row < a.N ? unit_bytes : 0u;
            const Row rx = row_of(a.x, row * row_bytes, bytes);
#pragma unroll
            for (int i = 0; i < VPL; ++i) load_unit<Tag>(rx, chunk[i], q.x[j][i]);
            if constexpr (RES) {
                const Row rr = row_of(a.r, row * row_bytes, bytes);
#pragma unroll
                for (int i = 0; i < VPL; ++i) load_unit<Tag>(rr, chunk[i], q.r[j][i]);
            }
        }
    };
    const int64_t first = (static_cast<int64_t>(blockIdx.x) * groups + group) * R, step = static_cast<int64_t>(a.nb) * groups * R;
    Rows bufs[kDepth];
#pragma unroll
    for (int d = 0; d < kDepth - 1; ++d) fetch(first + d * step, bufs[d]);
    const Row rw = row_of(a.w, 0, unit_bytes);
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        u32x4 t[NV];
        load_unit<Tag, 0>(rw, chunk[i], t);
        U::unpack(t, W[i]);
    }
    int buf = 0;
    const auto compute = [&](int64_t base, Rows& now) {
        float rs[R], big[R];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int64_t row = base + j;
            const Row rh = row_of(a.h, row * row_bytes, RES && row < a.N ? unit_bytes : 0u);
            float s = 0.0f;
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < VPL; ++i) {
                float v[8];
                if constexpr (RES) {
                    float rv[8];
                    U::unpack(now.x[j][i], v);
                    U::unpack(now.r[j][i], rv);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] += rv[e];
                    U::pack(v, now.x[j][i]);
                    store_unit<Tag>(rh, chunk[i], now.x[j][i]);
                }
                U::unpack(now.x[j][i], v);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    s += v[e] * v[e];
                    if constexpr (ROW) {
                        const uint32_t b = __builtin_bit_cast(uint32_t, v[e] * W[i][e]) & 0x7fffffffu;
                        top = b > top ? b : top;
                    }
                }
            }
            rs[j] = wave_sum(s);
            if constexpr (ROW) {
                top = row16_max(top);
                const uint32_t t0 = __builtin_amdgcn_readlane(top, 0), t1 = __builtin_amdgcn_readlane(top, 16);
                const uint32_t t2 = __builtin_amdgcn_readlane(top, 32), t3 = __builtin_amdgcn_readlane(top, 48);
                const uint32_t u = t0 > t1 ? t0 : t1, w = t2 > t3 ? t2 : t3;
                big[j] = __builtin_bit_cast(float, u > w ? u : w);
            }
        }
        if constexpr (K > 1) {
            if (lane == 0) {
#pragma unroll
                for (int j = 0; j < R; ++j) {
                    part[buf][j][wave][0] = rs[j];
                    if constexpr (ROW) part[buf][j][wave][1] = big[j];
                }
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < R; ++j) {
                float s = 0.0f;
                uint32_t top = 0;
#pragma unroll
                for (int w = 0; w < K; ++w) {
                    s += part[buf][j][w][0];
                    if constexpr (ROW) {
                        const uint32_t b = __builtin_bit_cast(uint32_t, part[buf][j][w][1]);
                        top = b > top ? b : top;
                    }
                }
                rs[j] = s;
                big[j] = __builtin_bit_cast(float, top);
            }
            buf ^= 1;
        }
#pragma unroll
        for (int j = 0; j < R; ++j) {
            rs[j] = rsqrtf(rs[j] * a.inv_D + a.eps);
#pragma unroll
            for (int i = 0; i < VPL; ++i) opaque(now.x[j][i]);
        }
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int64_t row = base + j;
            if (row < a.N) {
                store_float(row_of(a.rstd, row * 4, 4), first_lane, rs[j]);
                Scale sc;
                if constexpr (ROW) {
                    sc = scale_of<C>(__builtin_bit_cast(uint32_t, big[j] * rs[j]) & 0x7fffffffu);
                    if constexpr (!VALUES) store_float(row_of(a.scales, row * 4, 4), first_lane, sc.s);
                }
                const Row rout = VALUES ? row_of(a.out, row * row_bytes, unit_bytes)
                                        : row_of(a.out, row * a.D, static_cast<uint32_t>(a.D));
                const Row rcs = row_of(a.scales, row * a.groups * 4, VALUES ? 0u : static_cast<uint32_t>(a.groups) * 4u);
#pragma unroll
                for (int i = 0; i < VPL; ++i) {
                    float v[8];
                    U::unpack(now.x[j][i], v);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = (v[e] * rs[j]) * W[i][e];
                    if constexpr (!ROW) {
                        uint32_t top = 0;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const uint32_t b = __builtin_bit_cast(uint32_t, v[e]) & 0x7fffffffu;
                            top = b > top ? b : top;
                        }
                        // lanes beyond the row: 0, or NaN where rstd is NaN and so every v is
                        sc = scale_of<C>(group_max(top, a.lanes_log2));
                        if constexpr (!VALUES) store_float(rcs, scale_off[i], sc.s);
                    }
                    const u32x2 w = encode<C>(v, sc);
                    if constexpr (VALUES) {
                        u32x4 o[NV];
                        stand_for<Tag, C>(w, sc.s, v);
                        U::pack(v, o);
                        store_unit<Tag>(rout, chunk[i], o);
                    } else {
                        store_codes(rout, chunk[i], w, a.keep);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
    };
    for (int64_t base = first; base < a.N;) {
#pragma unroll
        for (int d = 0; d < kDepth; ++d) {
            if (base >= a.N) break;
            fetch(base + (kDepth - 1) * step, bufs[(d + kDepth - 1) % kDepth]);
            __builtin_amdgcn_sched_barrier(0);               // keep the requests up here
            compute(base, bufs[d]);
            base += step;
        }
    }
}

struct RmsqBwdArgs {
    const void* dy;
    const void* dh;
    const void* h;
    const void* w;
    const float* rstd;
    void* dx;
    void* dr;                // a second copy of dx, or null
    float* ws;               // [nb][D] fp32 partial dw sums
    int64_t N;
    int32_t nb;
    int32_t D;
    int32_t nchunks;
    float inv_D;
};

constexpr int rmsq_bwd_waves(int vpl, int nv, int r, bool dh) {
    return rmsq_waves(vpl * (16 + kDepth * r * 4 * nv * (dh ? 3 : 2)) + 56);
}

template <typename Tag, int VPL, int K, int R, bool DH>
__global__ __launch_bounds__(K* kWave* groups_most(K, rmsq_bwd_waves(VPL, Unit<Tag>::NV, R, DH)))
LNMOD_OCCUPANCY(rmsq_bwd_waves(VPL, Unit<Tag>::NV, R, DH))
void rmsq_bwd_kernel(const RmsqBwdArgs a) {
    using U = Unit<Tag>;
    constexpr int NV = U::NV;
    __shared__ float part[2][R][K];
    extern __shared__ f32x4 sums[];          // see add_groups
    const int lane = threadIdx.x & (kWave - 1);
    const int in_block = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave = K > 1 ? in_block : 0;   // of the row
    const int groups = K > 1 ? 1 : static_cast<int>(blockDim.x) >> 6, group = K > 1 ? 0 : in_block;
    const int64_t row_bytes = static_cast<int64_t>(a.D) * IO<Tag>::kBytes;
    const uint32_t unit_bytes = static_cast<uint32_t>(row_bytes);

    uint32_t chunk[VPL];
    float W[VPL][8], acc_all[1][VPL][8];
    float(&acc)[VPL][8] = acc_all[0];
    struct Rows {
        u32x4 dy[R][VPL][NV], h[R][VPL][NV], dh[DH ? R : 1][DH ? VPL : 1][NV];
        float rs[R];
    };
    const auto fetch = [&](int64_t base, Rows& q) {
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int64_t row = base + j;
            const bool live = row < a.N;
            q.rs[j] = live ? float_at(a.rstd, live ? row : a.N - 1) : 0.0f;
            const uint32_t bytes = live ? unit_bytes : 0u;
            const Row rdy = row_of(a.dy, row * row_bytes, bytes), rh = row_of(a.h, row * row_bytes, bytes);
#pragma unroll
            for (int i = 0; i < VPL; ++i) {
                load_unit<Tag>(rdy, chunk[i], q.dy[j][i]);
                load_unit<Tag>(rh, chunk[i], q.h[j][i]);
            }
            if constexpr (DH) {
                const Row rdh = row_of(a.dh, row * row_bytes, bytes);
#pragma unroll
                for (int i = 0; i < VPL; ++i) load_unit<Tag>(rdh, chunk[i], q.dh[j][i]);
            }
        }
    };
#pragma unroll
    for (int i = 0; i < VPL; ++i) chunk[i] = static_cast<uint32_t>((i * K + wave) * kWave + lane);
    const int64_t first = (static_cast<int64_t>(blockIdx.x) * groups + group) * R, step = static_cast<int64_t>(a.nb) * groups * R;
    Rows bufs[kDepth];
#pragma unroll
    for (int d = 0; d < kDepth - 1; ++d) fetch(first + d * step, bufs[d]);
    const Row rw = row_of(a.w, 0, unit_bytes);
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        u32x4 t[NV];
        load_unit<Tag, 0>(rw, chunk[i], t);
        U::unpack(t, W[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[i][e] = 0.0f;
    }
    int buf = 0;
    const auto compute = [&](int64_t base, Rows& now) {
        float c[R];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            float p = 0.0f;
#pragma unroll
            for (int i = 0; i < VPL; ++i) {
                float dyv[8], hv[8];
                U::unpack(now.dy[j][i], dyv);
                U::unpack(now.h[j][i], hv);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float t = dyv[e] * (hv[e] * now.rs[j]);
                    p += t * W[i][e];
                    acc[i][e] += t;
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) asm volatile("" : "+v"(acc[i][e]));     // pinned here (see ckpt_bwd_kernel)
                __builtin_amdgcn_sched_barrier(0);
            }
            c[j] = wave_sum(p);
        }
        if constexpr (K > 1) {
            if (lane == 0) {
#pragma unroll
                for (int j = 0; j < R; ++j) part[buf][j][wave] = c[j];
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < R; ++j) {
                float t = 0.0f;
#pragma unroll
                for (int w = 0; w < K; ++w) t += part[buf][j][w];
                c[j] = t;
            }
            buf ^= 1;
        }
#pragma unroll
        for (int j = 0; j < R; ++j) {
#pragma unroll
            for (int i = 0; i < VPL; ++i) {
                opaque(now.dy[j][i]);
                opaque(now.h[j][i]);
            }
        }
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int64_t row = base + j;
            const uint32_t bytes = row < a.N ? unit_bytes : 0u;
            const Row rdx = row_of(a.dx, row * row_bytes, bytes);
            const float k2 = now.rs[j] * (c[j] * a.inv_D);
#pragma unroll
            for (int i = 0; i < VPL; ++i) {
                float dyv[8], hv[8], o[8];
                U::unpack(now.dy[j][i], dyv);
                U::unpack(now.h[j][i], hv);
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = (dyv[e] * W[i][e]) * now.rs[j] - (hv[e] * now.rs[j]) * k2;
                if constexpr (DH) {
                    float t[8];
                    U::unpack(now.dh[j][i], t);
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] += t[e];
                }
                u32x4 t[NV];
                U::pack(o, t);
                store_unit<Tag>(rdx, chunk[i], t);
                if (a.dr) store_unit<Tag>(row_of(a.dr, row * row_bytes, bytes), chunk[i], t);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    for (int64_t base = first; base < a.N;) {
#pragma unroll
        for (int d = 0; d < kDepth; ++d) {
            if (base >= a.N) break;
            fetch(base + (kDepth - 1) * step, bufs[(d + kDepth - 1) % kDepth]);
            __builtin_amdgcn_sched_barrier(0);               // keep the requests up here
            compute(base, bufs[d]);
            base += step;
        }
    }
    add_groups<units_at_once(VPL, rmsq_bwd_waves(VPL, NV, R, DH))>(acc_all, group, groups, sums);
    const Row slot = row_of(a.ws, static_cast<int64_t>(blockIdx.x) * a.D * 4, group == 0 ? static_cast<uint32_t>(a.D) * 4u : 0u);
#pragma unroll
    for (int i = 0; i < VPL; ++i) store_sums8(slot, chunk[i], acc[i]);
}

}  // namespace lnmod
