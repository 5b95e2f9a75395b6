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
    // a product is kParts instructions, taken one after the other of several products: each waits for its sum's last one
    static constexpr int kParts = 2;
    __device__ static inline Sum add(const Frag& a, const Frag& b, Sum c, int h) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(a.v[h], b.v[h], c, 0, 0, 0);
    }
};

template <> struct Mac<e4m3_code, bf16_io> {
    typedef f32x4 Sum;
    typedef i32x8 Frag;
    __device__ static inline Sum zero() { return Sum{0.0f, 0.0f, 0.0f, 0.0f}; }
    __device__ static inline Frag frag(const i32x4& lo, const i32x4& hi) { return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7); }
    static constexpr int kParts = 1;
    __device__ static inline Sum add(const Frag& a, const Frag& b, Sum c, int) {
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
    static constexpr int kParts = 4;
    __device__ static inline Sum add(const Frag& a, const Frag& b, Sum c, int h) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a.v[h], b.v[h], c, 0, 0, 0);
    }
};

typedef uint8_t __attribute__((address_space(3))) lds_byte;

__device__ inline void wait_loads() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }

// Sixteen codes of a row of which `left` exist (a multiple of 8, or fewer than 1), the others 0.
__device__ inline u32x4 load_codes16(Row src, uint32_t offset, int uniform, int left) {
    u32x4 v = {0u, 0u, 0u, 0u};
    if (left >= 16) v = __builtin_amdgcn_raw_buffer_load_b128(src, offset, uniform, 0);
    else if (left > 0) {
        const u32x2 h = __builtin_amdgcn_raw_buffer_load_b64(src, offset, uniform, 0);
        v[0] = h[0];
        v[1] = h[1];
    }
    return v;
}

// Which tile a block computes.  Consecutive blocks go to the eight XCDs in turn, each with a cache of its own: an XCD gets a run
// of tiles, and inside it eight rows of tiles are walked side by side, so that the tiles that its CUs have in hand at a time
// share their rows of a and of w.
struct Tile {
    uint32_t m, n;
};
__device__ inline Tile tile_of(const ProductArgs& a, uint32_t id) {
    const uint32_t x = id % kXcds, seq = x * a.each + (x < a.more ? x : a.more) + id / kXcds;
    const uint32_t band = a.band_of(seq), at = seq - band * kBandRows * a.tiles_n;
    const uint32_t left = a.tiles_m - band * kBandRows, rows = left < kBandRows ? left : kBandRows;
    const uint32_t n = left < kBandRows ? a.row_of(at) : at / kBandRows;
    return Tile{band * kBandRows + at - n * rows, n};
}

// What the outputs of a wave's TM x TN fragments, the first of them at (m0, n0), are scaled with.  A lane holds eight
// consecutive outputs of a row for each pair of fragments of w, four lanes 32.
template <typename Tag, int TM, int TN>
struct Scales {
    static constexpr bool kHalf = std::is_same<Tag, bf16_io>::value;
    float a[TM], w[TN / 2][8];
    u32x4 b[TN / 2][Unit<Tag>::NV];
    // m0 and n0 are uniform; rows and features beyond the last one have the last one's
    __device__ inline void load(const ProductArgs& p, int64_t m0, int64_t n0) {
        constexpr int kBytes = IO<Tag>::kBytes;
        const int lane = threadIdx.x & (kWave - 1);
        const int rows = static_cast<int>(p.M - 1 - m0 < TM * 16 ? p.M - 1 - m0 : TM * 16);
        const int most = static_cast<int>(p.N - 1 - n0 < TN * 16 ? p.N - 1 - n0 : TN * 16);
        const Row ra = row_of(p.sa, m0 * 4, 0x7fffffffu), rw = row_of(p.sw, n0 * 4, 0x7fffffffu);
        const Row rb = row_of(p.bias, n0 * kBytes, 0x7fffffffu);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int m = i * 16 + (lane & 15);
            a[i] = load_float(ra, (m < rows ? m : rows) * 4);
        }
        if (p.N % 8 == 0) {                  // eight at a time, whatever they are aligned to
#pragma unroll
            for (int j = 0; j < TN / 2; ++j) {
                int n = j * 32 + (lane >> 4) * 8;
                if (n > most) n = most - 7;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const f32x4 t = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, n * 4 + 16 * h, 0, 0));
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[j][4 * h + e] = t[e];
                }
                if (!p.bias) continue;
#pragma unroll
                for (int h = 0; h < Unit<Tag>::NV; ++h) b[j][h] = __builtin_amdgcn_raw_buffer_load_b128(rb, n * kBytes + 16 * h, 0, 0);
            }
            return;
        }
#pragma unroll
        for (int j = 0; j < TN / 2; ++j) {
            float v[8] = {};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                int n = j * 32 + (lane >> 4) * 8 + e;
                if (n > most) n = most;
                w[j][e] = load_float(rw, n * 4);
                if (!p.bias) continue;
                if constexpr (kHalf) v[e] = __builtin_bit_cast(float, static_cast<uint32_t>(__builtin_amdgcn_raw_buffer_load_b16(rb, n * 2, 0, 0)) << 16);
                else v[e] = load_float(rb, n * 4);
            }
            Unit<Tag>::pack(v, b[j]);
        }
    }
};

// Where every row of y starts at a multiple of eight outputs they are stored as they lie in the lanes.
template <typename C, typename Tag, int TM, int TN>
__device__ inline void store_products(const ProductArgs& p, const typename Mac<C, Tag>::Sum (&acc)[TM][TN], const Scales<Tag, TM, TN>& s,
                                      int64_t m0, int64_t n0) {
    constexpr bool kHalf = std::is_same<Tag, bf16_io>::value;
    const int lane = threadIdx.x & (kWave - 1);
    const bool whole = p.N % 8 == 0;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t m = m0 + i * 16 + (lane & 15);
#pragma unroll
        for (int j = 0; j < TN / 2; ++j) {
            const int64_t n = n0 + j * 32 + (lane >> 4) * 8;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(acc[i][2 * j + e / 4][e % 4]) * s.a[i] * s.w[j][e];
            if (p.bias) {
                float b[8];
                Unit<Tag>::unpack(s.b[j], b);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += b[e];
            }
            if (m >= p.M || n >= p.N) continue;
            if (whole) {
                char* y = static_cast<char*>(p.y) + (m * p.N + n) * IO<Tag>::kBytes;
                u32x4 q[kHalf ? 1 : 2];
                if constexpr (kHalf) q[0] = IO<Tag>::pack(v);
                else Unit<f32_io>::pack(v, q);
#pragma unroll
                for (int h = 0; h < (kHalf ? 1 : 2); ++h) {
                    u32x4* to = reinterpret_cast<u32x4*>(y) + h;
                    if (p.keep) *to = q[h];
                    else __builtin_nontemporal_store(q[h], to);
                }
                continue;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (n + e >= p.N) continue;
                if constexpr (kHalf) static_cast<__bf16*>(p.y)[m * p.N + n + e] = static_cast<__bf16>(v[e]);
                else static_cast<float*>(p.y)[m * p.N + n + e] = v[e];
            }
        }
    }
}

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
    const uint32_t id = blockIdx.y * gridDim.x + blockIdx.x;
    if (id >= a.tiles) return;
    const Tile tile = tile_of(a, id);
    const int64_t m0 = static_cast<int64_t>(tile.m) * BM, n0 = static_cast<int64_t>(tile.n) * BN;
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
            for (int i = 0; i < count; ++i)
                *reinterpret_cast<u32x4*>(dst + (i * NW + wave) * 1024 + lane * 16) = load_codes16(src, off[i], k0, left);
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
            for (int h = 0; h < mac::kParts; ++h)
#pragma unroll
                for (int i = 0; i < TM; ++i) acc[i][j] = mac::add(wf, xf[i], acc[i][j], h);
        }
        __syncthreads();
    }

    Scales<Tag, TM, TN> scales;
    scales.load(a, m0 + wm * TM * 16, n0 + wn * TN * 16);
    store_products<C, Tag, TM, TN>(a, acc, scales, m0 + wm * TM * 16, n0 + wn * TN * 16);
}

// ---- large products ------------------------------------------------------------------------------------------------
// 1024 bytes from global memory into LDS, sixteen from each lane's address, at dst + 16 lane.  In assembly because the compiler
// makes every later read of LDS wait for such a load, whatever part of LDS it fills: no register is written here, and whoever
// reads dst has waited for this wave's vmcnt and met the others at a barrier first.
__device__ inline void load_lds(Row src, uint32_t offset, int uniform, const uint8_t* dst) {
    const uint32_t at = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_byte*)dst)));
    asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds" ::"v"(offset), "s"(src), "s"(uniform), "s"(at) : "m0");
}

// 256 x 256 outputs by eight waves of 128 x 64, two on each SIMD that take turns: while one reads the fragments of its next 128
// features from LDS and sends for the features after them, the other multiplies.  Waves 0 to 3 bring a, one step ahead into
// two buffers, waves 4 to 7 w, two steps ahead into three.
//
//   phase      2t                                  2t + 1                               2t + 2
//   waves 0-3  read a(t), w(t); send for a(t+1)    multiply t; wait                     read a(t+1), w(t+1); ...
//   waves 4-7  multiply t-1; wait                  read a(t), w(t); send for w(t+2)     multiply t; wait
//
// A block takes tiles until there are none, and the steps of all of them are one sequence: the next tile's first steps are sent
// for in the last steps of this one, whose outputs are stored in front of the next reading phase.  There are two steps to a
// tile at least.
template <typename C, typename Tag>
__global__ __launch_bounds__(8 * kWave, 2) void product_large_kernel(const ProductArgs a) {
    using mac = Mac<C, Tag>;
    constexpr int BM = 256, BN = 256, TM = 8, TN = 4, kPieces = 8, kPart = 256 * kBlockK;
    __shared__ __attribute__((aligned(1024))) uint8_t sx[2 * kPart], sw[3 * kPart];
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave & 1, wn = wave >> 1;
    const bool second = wave >= 4;                             // waves w and w + 4 share a SIMD
    const int K = a.K, whole = K / kBlockK, steps = (K + kBlockK - 1) / kBlockK;

    // what a lane brings: sixteen features of a row of each of eight pieces of eight rows; the sixteens of a row are exchanged
    // by the row, so that the eight rows that a fragment's lanes read at a time lie in different banks.  Rows beyond the last
    // one are the last one.
    const int c = (lane & 7) ^ (lane >> 3), quarter = wave & 3, slot = quarter * 8 + (lane >> 3);
    const int row = second ? ((slot >> 2) & 3) * 8 + ((slot >> 4) & 1) * 4 + (slot & 3) : slot;
    const uint32_t first = static_cast<uint32_t>(row) * K + c * 16;
    struct Source {
        int64_t at;                                            // of the tile's first row
        uint32_t last;                                         // a lane's offset in the last row that it may read
    };
    auto source = [&](const Tile& t) __attribute__((always_inline)) {
        const int64_t r0 = static_cast<int64_t>(second ? t.n : t.m) * 256, left = (second ? a.N : a.M) - 1 - r0;
        return Source{r0 * K, static_cast<uint32_t>(left < 255 ? left : 255) * K + c * 16};
    };
    const void* matrix = second ? a.w : a.a;
    auto bring = [&](const Source& s, uint8_t* to, int t) __attribute__((always_inline)) {
        const Row src = row_of(matrix, s.at, 0x7fffffffu);
        uint32_t off0 = first;
        asm volatile("" : "+v"(off0));                         // the addresses are formed here, not kept in registers across the loop
        if (t < whole) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const uint32_t off = off0 + i * 32 * K;
                load_lds(src, off < s.last ? off : s.last, t * kBlockK, to + (i * 4 + quarter) * 1024);
            }
        } else {
            const int left = K - t * kBlockK - c * 16;         // codes of this lane's sixteen that exist: a multiple of 8
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const uint32_t off = off0 + i * 32 * K;
                *reinterpret_cast<u32x4*>(to + (i * 4 + quarter) * 1024 + lane * 16) = load_codes16(src, off < s.last ? off : s.last, t * kBlockK, left);
            }
        }
    };

    const int fo = (lane & 15) * kBlockK + (((lane >> 4) ^ (lane & 7)) << 4);
    auto frag = [&](const uint8_t* p) __attribute__((always_inline)) {
        return mac::frag(*reinterpret_cast<const i32x4*>(p + fo), *reinterpret_cast<const i32x4*>(p + (fo ^ 64)));
    };

    uint32_t id = blockIdx.x;
    Tile tile = tile_of(a, id), next = tile;
    Source here = source(tile), there = here;
    const int ahead = second ? 2 : 1;
    bring(here, second ? sw : sx, 0);
    if (second) bring(here, sw + kPart, 1);
    wait_loads();
    __builtin_amdgcn_s_barrier();
    if (second) __builtin_amdgcn_s_barrier();
    int odd = 0, at = 0;                                       // the step's buffers, its number modulo 2 and 3
#pragma unroll 1
    while (true) {
        id += gridDim.x;
        const bool more = id < a.tiles;
        if (more) {
            next = tile_of(a, id);
            there = source(next);
        }
        typename mac::Sum acc[TM][TN];
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = mac::zero();
        Scales<Tag, TM, TN> scales;
        const int64_t m = static_cast<int64_t>(tile.m) * BM + wm * TM * 16, n = static_cast<int64_t>(tile.n) * BN + wn * TN * 16;

        auto step = [&](int t) __attribute__((always_inline)) {
            typename mac::Frag xf[TM], wf[TN];
            const uint8_t *px = sx + odd * kPart + wm * TM * 16 * kBlockK, *pw = sw + at * kPart + wn * TN * 16 * kBlockK;
#pragma unroll
            for (int j = 0; j < TN; ++j) wf[j] = frag(pw + j * 16 * kBlockK);
#pragma unroll
            for (int i = 0; i < TM; ++i) xf[i] = frag(px + i * 16 * kBlockK);
            __builtin_amdgcn_sched_barrier(0);
            uint8_t* to = second ? sw + (at == 0 ? 2 : at - 1) * kPart : sx + (odd ^ 1) * kPart;
            if (t + ahead < steps) bring(here, to, t + ahead);
            else if (more) bring(there, to, t + ahead - steps);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int i = 0; i < TM; ++i) {
#pragma unroll
                for (int h = 0; h < mac::kParts; ++h)
#pragma unroll
                    for (int j = 0; j < TN; ++j) acc[i][j] = mac::add(wf[j], xf[i], acc[i][j], h);
            }
            __builtin_amdgcn_s_setprio(0);
            __builtin_amdgcn_sched_barrier(0);
            wait_loads();
            __builtin_amdgcn_s_barrier();
            at = at == 2 ? 0 : at + 1;
            odd ^= 1;
        };
#pragma unroll 1
        for (int t = 0; t < steps; ++t) step(t);
        scales.load(a, m, n);
        store_products<C, Tag, TM, TN>(a, acc, scales, m, n);
        if (!more) break;
        tile = next;
        here = there;
    }
    if (!second) __builtin_amdgcn_s_barrier();
}

}  // namespace lnmod
