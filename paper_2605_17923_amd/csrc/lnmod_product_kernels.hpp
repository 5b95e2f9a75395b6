// lnmod_product_kernels.hpp -- gfx950 device code of the product of 8-bit codes that have one scale for each row.
//
//   y[m,n] = (sum_k a[m,k] w[n,k]) sa[m] sw[n] + bias[n]
#pragma once
#include "lnmod_code.hpp"

namespace lnmod {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kBlockK = 128;                 // features of a step: one cache line of a row

// Sums and products of sixteen rows of each operand.  A lane holds 32 codes of one row: features 16 (lane / 16) .. + 15 of
// the first and of the second half of a step.  Which feature goes where is no matter as long as both operands agree.
//
// int8 sums are whole numbers and exact.  The matrix instruction for e4m3 adds the products of eight neighbouring features with
// 13 bits below the largest of them and drops the rest (measured: 2^-13 of 2^16 survives beside it, 2^-14 does not; between
// such eights, and to the running sum, it keeps 24 bits).  So y is off by less than 7 * 2^-13 of the sum over the eights of
// their largest product: on normal values 1.5e-5 of y's root mean square, 5e-5 with outliers, against 1.7e-3 for the rounding of
// y to bf16.  Where y is float32 that would be the largest error by far, so there the codes go to half precision (exactly)
// and through that type's instruction, which keeps 24 bits, at half the rate.
template <typename C, typename Tag> struct Mac;

template <typename Tag> struct Mac<int8_code, Tag> {
    typedef i32x4 Sum;
    struct Frag {
        i32x4 v[2];
    };
    __device__ static inline Sum zero() { return Sum{0, 0, 0, 0}; }
    __device__ static inline Frag frag(const i32x4& lo, const i32x4& hi) { return Frag{{lo, hi}}; }
    __device__ static inline Sum add(const Frag& a, const Frag& b, Sum c) {
        c = __builtin_amdgcn_mfma_i32_16x16x64_i8(a.v[0], b.v[0], c, 0, 0, 0);
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(a.v[1], b.v[1], c, 0, 0, 0);
    }
};

template <> struct Mac<e4m3_code, bf16_io> {
    typedef f32x4 Sum;
    typedef i32x8 Frag;
    __device__ static inline Sum zero() { return Sum{0.0f, 0.0f, 0.0f, 0.0f}; }
    __device__ static inline Frag frag(const i32x4& lo, const i32x4& hi) { return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7); }
    __device__ static inline Sum add(const Frag& a, const Frag& b, Sum c) {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, 0, 0, 0);
    }
};

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

template <> struct Mac<e4m3_code, f32_io> {
    typedef f32x4 Sum;
    struct Frag {
        f16x8 v[4];
    };
    __device__ static inline Sum zero() { return Sum{0.0f, 0.0f, 0.0f, 0.0f}; }
    __device__ static inline f16x8 halves(int a, int b) {
        const f16x2 p = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, false), q = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, true);
        const f16x2 r = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, false), s = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, true);
        return f16x8{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
    }
    __device__ static inline Frag frag(const i32x4& lo, const i32x4& hi) {
        return Frag{{halves(lo[0], lo[1]), halves(lo[2], lo[3]), halves(hi[0], hi[1]), halves(hi[2], hi[3])}};
    }
    __device__ static inline Sum add(const Frag& a, const Frag& b, Sum c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x32_f16(a.v[i], b.v[i], c, 0, 0, 0);
        return c;
    }
};

typedef uint8_t __attribute__((address_space(3))) lds_byte;

// BM x BN outputs per block of WM x WN waves.
template <typename C, typename Tag, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM* WN* kWave, 1) void product_tile_kernel(const ProductArgs a) {
    constexpr int NW = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr int XI = BM / 8 / NW, WI = BN / 8 / NW;          // loads of a wave for each operand and step
    static_assert(TN % 2 == 0 && XI * 8 * NW == BM && WI * 8 * NW == BN, "tile");
    __shared__ __attribute__((aligned(1024))) uint8_t sx[2][BM * kBlockK], sw[2][BN * kBlockK];

    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;
    const int64_t tile = static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x;
    if (tile >= a.tiles) return;
    const int64_t m0 = tile % a.tiles_m * BM, n0 = tile / a.tiles_m * BN;
    const int K = a.K, steps = (K + kBlockK - 1) / kBlockK;

    // what a lane fetches: row slot (i*NW + wave)*8 + lane/8, sixteen features; the slot of eight sixteens is permuted by
    // the row, so that eight consecutive rows of a fragment lie in different banks
    const int c = (lane & 7) ^ (lane >> 3);
    uint32_t xo[XI], wo[WI];
#pragma unroll
    for (int i = 0; i < XI; ++i) {
        int64_t r = (i * NW + wave) * 8 + (lane >> 3);
        if (m0 + r >= a.M) r = a.M - 1 - m0;
        xo[i] = static_cast<uint32_t>(r) * K + c * 16;
    }
#pragma unroll
    for (int i = 0; i < WI; ++i) {
        const int slot = (i * NW + wave) * 8 + (lane >> 3);
        int64_t r = (slot & ~31) + ((slot >> 2) & 3) * 8 + ((slot >> 4) & 1) * 4 + (slot & 3);
        if (n0 + r >= a.N) r = a.N - 1 - n0;
        wo[i] = static_cast<uint32_t>(r) * K + c * 16;
    }
    const Row xrow = row_of(a.a, m0 * K, 0x7fffffffu), wrow = row_of(a.w, n0 * K, 0x7fffffffu);

    auto fetch = [&](Row src, const uint32_t* off, int count, uint8_t* dst, int t) {
        const int k0 = t * kBlockK;
        if (k0 + kBlockK <= K) {
            for (int i = 0; i < count; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (lds_byte*)(dst + (i * NW + wave) * 1024), 16, off[i], k0, 0, 0);
        } else {
            const int left = K - k0 - c * 16;                  // codes of this lane's sixteen that exist: a multiple of 8
            for (int i = 0; i < count; ++i) {
                u32x4 v = {0u, 0u, 0u, 0u};
                if (left >= 16) v = __builtin_amdgcn_raw_buffer_load_b128(src, off[i], k0, 0);
                else if (left > 0) {
                    const u32x2 h = __builtin_amdgcn_raw_buffer_load_b64(src, off[i], k0, 0);
                    v[0] = h[0];
                    v[1] = h[1];
                }
                *reinterpret_cast<u32x4*>(dst + (i * NW + wave) * 1024 + lane * 16) = v;
            }
        }
    };

    using mac = Mac<C, Tag>;
    typename mac::Sum acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = mac::zero();

    const int fo = (lane & 15) * kBlockK + (((lane >> 4) ^ (lane & 7)) << 4);
    for (int t = 0; t < steps; ++t) {
        fetch(xrow, xo, XI, sx[0], t);
        fetch(wrow, wo, WI, sw[0], t);
        __syncthreads();
        typename mac::Frag xf[TM];
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const uint8_t* p = sx[0] + (wm * TM + i) * 16 * kBlockK;
            xf[i] = mac::frag(*reinterpret_cast<const i32x4*>(p + fo), *reinterpret_cast<const i32x4*>(p + (fo ^ 64)));
        }
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const uint8_t* p = sw[0] + (wn * TN + j) * 16 * kBlockK;
            const typename mac::Frag wf = mac::frag(*reinterpret_cast<const i32x4*>(p + fo), *reinterpret_cast<const i32x4*>(p + (fo ^ 64)));
#pragma unroll
            for (int i = 0; i < TM; ++i) acc[i][j] = mac::add(wf, xf[i], acc[i][j]);
        }
        __syncthreads();
    }

    // eight consecutive outputs of a row in a lane, for each pair of fragments of w
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t m = m0 + (wm * TM + i) * 16 + (lane & 15);
        if (m >= a.M) continue;
        const float sa = a.sa[m];
#pragma unroll
        for (int j = 0; j < TN; j += 2) {
            const int64_t n = n0 + (wn * TN + j) * 16 + (lane >> 4) * 8;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (n + e >= a.N) continue;
                float v = static_cast<float>(acc[i][j + e / 4][e % 4]) * sa * a.sw[n + e];
                if constexpr (std::is_same<Tag, bf16_io>::value) {
                    if (a.bias) v += static_cast<float>(static_cast<const __bf16*>(a.bias)[n + e]);
                    static_cast<__bf16*>(a.y)[m * a.N + n + e] = static_cast<__bf16>(v);
                } else {
                    if (a.bias) v += static_cast<const float*>(a.bias)[n + e];
                    static_cast<float*>(a.y)[m * a.N + n + e] = v;
                }
            }
        }
    }
}

}  // namespace lnmod
