// lnmod_product_kernels.hpp -- gfx950 device code of the product of 8-bit codes that have one scale for each row.
//
//   y[m,n] = (sum_k a[m,k] w[n,k]) sa[m] sw[n] + bias[n]
//
// Three kernels, by what bounds a product (lnmod_product_plan.hpp picks).  A few rows read w once: HBM, and the 2 to 3 us that a launch
// and a chain of loads take.  Products of some hundred rows or features have few tiles, and each step of a tile waits for the
// caches: small tiles, several steps on their way, teams of waves that share out the sum.  Large ones are bound by the matrix
// instructions and by what LDS gives them, 256 x 256 outputs a block.
//
// A step is 128 features of rows of a and of w, one cache line of each, brought straight to LDS.  The sixteen rows of w that a
// fragment takes are chosen so that a lane ends up with eight neighbouring outputs: one store of 16 bytes in bf16.
#pragma once
#include "lnmod_code.hpp"
#include "lnmod_product_plan.hpp"

namespace lnmod {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

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

// A barrier that no access to memory is moved across.
__device__ inline void meet() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
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
    // m0 and n0 are uniform, and there are outputs (has_outputs); rows and features beyond the last one have the last one's
    __device__ inline void load_rows(const ProductArgs& p, int64_t m0) {
        const int lane = threadIdx.x & (kWave - 1);
        const int last = last_of(p.M, m0, TM * 16);
        const Row ra = row_of(p.sa, m0 * 4, 0x7fffffffu);
#pragma unroll
        for (int i = 0; i < TM; ++i) a[i] = load_float(ra, held(i * 16 + (lane & 15), last) * 4);
    }
    // of the pairs of fragments from `from` to `to` - 1
    __device__ inline void load_features(const ProductArgs& p, int64_t n0, int from, int to) {
        constexpr int kBytes = IO<Tag>::kBytes;
        const int lane = threadIdx.x & (kWave - 1);
        const int last = last_of(p.N, n0, TN * 16);
        const Row rw = row_of(p.sw, n0 * 4, 0x7fffffffu), rb = row_of(p.bias, n0 * kBytes, 0x7fffffffu);
#pragma unroll
        for (int j = from; j < to; ++j) {
            const int n = j * 32 + (lane >> 4) * 8;
            if (p.wide && n + 7 <= last) {   // eight at a time, whatever they are aligned to
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const f32x4 t = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, n * 4 + 16 * h, 0, 0));
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[j][4 * h + e] = t[e];
                }
                if (!p.bias) continue;
#pragma unroll
                for (int h = 0; h < Unit<Tag>::NV; ++h) b[j][h] = __builtin_amdgcn_raw_buffer_load_b128(rb, n * kBytes + 16 * h, 0, 0);
                continue;
            }
            float v[8] = {};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int at = held(n + e, last);
                w[j][e] = load_float(rw, at * 4);
                if (!p.bias) continue;
                if constexpr (kHalf) v[e] = __builtin_bit_cast(float, static_cast<uint32_t>(__builtin_amdgcn_raw_buffer_load_b16(rb, at * 2, 0, 0)) << 16);
                else v[e] = load_float(rb, at * 4);
            }
            Unit<Tag>::pack(v, b[j]);
        }
    }
};

// sum * sa * sw.  A sum is 0 or 2^-18 (e4m3's smallest code squared) to 2^35 in magnitude, so with a plain sa the first product is a normal
// float and the two are formed from left to right.  Beyond (a row of activations with a largest value above 6e29, or below
// 2^-100) the mantissas are multiplied and the exponents added, which rounds where those two products would and goes beyond float32 only
// where y does.  A wave with such a scale takes a copy of the stores of its own: 32 760 x 5120 by 15 360 int8 1974 us before there was
// one, 1976 with it, 2004 with both ways in one loop; 1943 with every second row so, 1902 before.
__device__ inline bool plain_scale(float sa) { return __builtin_fabsf(sa) >= 0x1p-108f && __builtin_fabsf(sa) < 0x1p92f; }
__device__ inline float far_scaled(float sum, float sa, float sw) {
    return __builtin_ldexpf(sum * __builtin_amdgcn_frexp_mantf(sa) * __builtin_amdgcn_frexp_mantf(sw),
                            __builtin_amdgcn_frexp_expf(sa) + __builtin_amdgcn_frexp_expf(sw));
}

// Eight outputs of a lane are stored at once, at any element's address; those of the last features one by one.
template <bool FAR, typename C, typename Tag, int TM, int TN>
__device__ inline void store_scaled(const ProductArgs& p, const typename Mac<C, Tag>::Sum (&acc)[TM][TN], Scales<Tag, TM, TN>& s, int64_t m0,
                                    int64_t n0) {
    constexpr bool kHalf = std::is_same<Tag, bf16_io>::value;
    const int lane = threadIdx.x & (kWave - 1);
#pragma unroll
    for (int j = 0; j < TN / 2; ++j) {
        if (!kHalf && j > 0) s.load_features(p, n0, j, j + 1);       // float32 biases of all pairs at once would not fit beside the sums
        const int64_t n = n0 + j * 32 + (lane >> 4) * 8;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int64_t m = m0 + i * 16 + (lane & 15);
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float sum = static_cast<float>(acc[i][2 * j + e / 4][e % 4]);
                v[e] = FAR ? far_scaled(sum, s.a[i], s.w[j][e]) : sum * s.a[i] * s.w[j][e];
            }
            if (p.bias) {
                float b[8];
                Unit<Tag>::unpack(s.b[j], b);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += b[e];
            }
            if (m >= p.M || n >= p.N) continue;
            if (n + 8 <= p.N) {
                typedef u32x4 loose __attribute__((aligned(2)));
                loose* y = reinterpret_cast<loose*>(static_cast<char*>(p.y) + (m * p.N + n) * IO<Tag>::kBytes);
                u32x4 q[Unit<Tag>::NV];
                Unit<Tag>::pack(v, q);
#pragma unroll
                for (int h = 0; h < Unit<Tag>::NV; ++h) {
                    if (p.keep) y[h] = q[h];
                    else __builtin_nontemporal_store(q[h], y + h);
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

template <typename C, typename Tag, int TM, int TN>
__device__ inline void store_products(const ProductArgs& p, const typename Mac<C, Tag>::Sum (&acc)[TM][TN], int64_t m0, int64_t n0) {
    if (!has_outputs(p, m0, n0)) return;
    Scales<Tag, TM, TN> s;
    s.load_rows(p, m0);
    s.load_features(p, n0, 0, std::is_same<Tag, bf16_io>::value ? TN / 2 : 1);      // on their way while the rows' scales are looked at
    bool plain = true;
#pragma unroll
    for (int i = 0; i < TM; ++i) plain = plain & plain_scale(s.a[i]);
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(!plain) == 0, 1)) store_scaled<false, C, Tag, TM, TN>(p, acc, s, m0, n0);
    else store_scaled<true, C, Tag, TM, TN>(p, acc, s, m0, n0);
}

// 1024 bytes from global memory into LDS, sixteen from each lane's address, at dst + 16 lane.  In assembly because the compiler
// makes every later read of LDS wait for such a load, whatever part of LDS it fills: no register is written here, and whoever
// reads dst has waited for this wave's vmcnt and met the others at a barrier first.
__device__ inline void load_lds(Row src, uint32_t offset, int uniform, const uint8_t* dst) {
    const uint32_t at = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_byte*)dst)));
    asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds" ::"v"(offset), "s"(src), "s"(uniform), "s"(at) : "m0");
}

// ---- ordinary products ---------------------------------------------------------------------------------------------
// BM x BN outputs per block: GROUPS teams of WM x WN waves, each of which takes every GROUPS-th step, has STAGES of them in LDS, of
// which one is multiplied while the others are on their way, and adds its sums to the first team's at the end.
//
// What bounds it is the way from the caches: a CU has one block or two, and a step lasts as long as its lines need, however
// small the tile (0.33 to 0.86 us, lnmod_product_plan.hpp).  So the lines of several steps are on their way at a time, teams take
// steps side by side, and the tile is the smallest that still fills the CUs: 1025 x 2600 by 1433 to float32 13.5 us (45 in
// tiles of the first kernel, 128 x 128), 96 x 4096 by 12 288 e4m3 12.1 us (50).  Both are with w in the last-level cache; from HBM 16.2
// and 17.3 us, the latter 3.1 TB/s.
template <typename C, typename Tag, int BM, int BN, int WM, int WN, int STAGES, int GROUPS>
__global__ __launch_bounds__(GROUPS* WM* WN* kWave) void product_tile_kernel(const ProductArgs a) {
    using mac = Mac<C, Tag>;
    constexpr int NW = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr int kPieces = (BM + BN) / 8 / NW, kStage = (BM + BN) * kBlockK;
    static_assert(TN % 2 == 0 && kPieces * 8 * NW == BM + BN && BM % 8 == 0 && STAGES >= 2, "tile");
    __shared__ __attribute__((aligned(1024))) uint8_t shared[GROUPS * STAGES * kStage];
    const uint32_t id = blockIdx.y * gridDim.x + blockIdx.x;
    if (id >= a.tiles) return;
    const Tile tile = tile_of(a, id);
    const int64_t m0 = static_cast<int64_t>(tile.m) * BM, n0 = static_cast<int64_t>(tile.n) * BN;

    const int lane = threadIdx.x & (kWave - 1);
    const int group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / NW, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % NW;
    const int wm = wave % WM, wn = wave / WM;
    uint8_t* stage = shared + group * STAGES * kStage;         // rows of w, then rows of a
    const int K = a.K, whole = K / kBlockK, steps = (K + kBlockK - 1) / kBlockK;

    // what a lane brings: piece i*NW + wave has eight rows, of which a lane has sixteen features of one; the sixteens of a row
    // are exchanged by the row, so that the eight rows that a fragment's lanes read at a time lie in different banks.  Rows
    // beyond the last one are the last one.
    const int c = (lane & 7) ^ (lane >> 3);
    uint32_t off[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        const int slot = (i * NW + wave) * 8 + (lane >> 3);
        int64_t r = slot - BN, most = a.M - 1 - m0;
        if (slot < BN) {
            r = (slot & ~31) + ((slot >> 2) & 3) * 8 + ((slot >> 4) & 1) * 4 + (slot & 3);
            most = a.N - 1 - n0;
        }
        off[i] = static_cast<uint32_t>(r < most ? r : most) * K + c * 16;
    }
    const Row xrow = row_of(a.a, m0 * K, 0x7fffffffu), wrow = row_of(a.w, n0 * K, 0x7fffffffu);
    auto bring = [&](uint8_t* to, int t) __attribute__((always_inline)) {
        if (t < whole) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
                load_lds((i * NW + wave) * 8 < BN ? wrow : xrow, off[i], t * kBlockK, to + (i * NW + wave) * 1024);
        } else if (t < steps) {
            const int left = K - t * kBlockK - c * 16;         // codes of this lane's sixteen that exist: a multiple of 8
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
                *reinterpret_cast<u32x4*>(to + (i * NW + wave) * 1024 + lane * 16) =
                    load_codes16((i * NW + wave) * 8 < BN ? wrow : xrow, off[i], t * kBlockK, left);
        }
    };

    typename mac::Sum acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = mac::zero();
    const int fo = (lane & 15) * kBlockK + (((lane >> 4) ^ (lane & 7)) << 4);
    auto frag = [&](const uint8_t* p) __attribute__((always_inline)) {
        return mac::frag(*reinterpret_cast<const i32x4*>(p + fo), *reinterpret_cast<const i32x4*>(p + (fo ^ 64)));
    };

#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) bring(stage + i * kStage, i * GROUPS + group);
    int at = 0, to = STAGES - 1;                               // the buffers of this step and of the one that is sent for
#pragma unroll 1
    for (int t0 = 0; t0 < steps; t0 += GROUPS) {
        const int t = t0 + group;
        // loads come back in their order: with the whole steps behind t still on their way, t is here
        if (t + (STAGES - 2) * GROUPS < whole) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kPieces * (STAGES - 2)) : "memory");
        else wait_loads();
        meet();                          // and every wave is done with the buffer that is filled now
        bring(stage + to * kStage, t + (STAGES - 1) * GROUPS);
        const uint8_t *pw = stage + at * kStage + wn * TN * 16 * kBlockK, *px = stage + at * kStage + (BN + wm * TM * 16) * kBlockK;
        if (GROUPS == 1 || t < steps) {
            typename mac::Frag xf[TM];
#pragma unroll
            for (int i = 0; i < TM; ++i) xf[i] = frag(px + i * 16 * kBlockK);
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const typename mac::Frag wf = frag(pw + j * 16 * kBlockK);
#pragma unroll
                for (int h = 0; h < mac::kParts; ++h)
#pragma unroll
                    for (int i = 0; i < TM; ++i) acc[i][j] = mac::add(wf, xf[i], acc[i][j], h);
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // its reads are done when it meets the others
        at = at == STAGES - 1 ? 0 : at + 1;
        to = to == STAGES - 1 ? 0 : to + 1;
    }
    if constexpr (GROUPS > 1) {
        typedef typename mac::Sum Sum;
        static_assert((GROUPS - 1) * BM * BN * 4 <= GROUPS * STAGES * kStage, "sums");
        Sum* sums = reinterpret_cast<Sum*>(shared) + wave * kWave + lane;
        constexpr int kEach = NW * kWave;                      // of a fragment, all waves of a team
        meet();
        if (group > 0) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) sums[((group - 1) * TM * TN + i * TN + j) * kEach] = acc[i][j];
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        meet();
        if (group > 0) return;
#pragma unroll
        for (int g = 0; g < GROUPS - 1; ++g)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] += sums[(g * TM * TN + i * TN + j) * kEach];
    }
    store_products<C, Tag, TM, TN>(a, acc, m0 + wm * TM * 16, n0 + wn * TN * 16);
}

// ---- few rows --------------------------------------------------------------------------------------------------------
// Up to 16 rows of a: w is read once, straight into registers, and that takes all the time there is.  A block has 16 features of
// y; its waves share out the steps and add their sums in LDS, wave by wave.  In a graph of such calls, int8, with w in the last-level
// cache and from HBM: 1 x 1536 by 1536 2.8 and 3.7 us, 16 x 2048 by 4096 3.7 and 4.8, 1 x 4096 by 4096 4.7 and 6.1.
constexpr int kFewWaves = 8, kFewDepth = 2, kFewOutputs = 16;

template <typename C, typename Tag>
__global__ __launch_bounds__(kFewWaves* kWave) void product_few_kernel(const ProductArgs a) {
    using mac = Mac<C, Tag>;
    typedef typename mac::Sum Sum;
    __shared__ Sum part[kFewWaves][kWave];
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int K = a.K, whole = K / kBlockK;
    const int64_t n0 = (static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x) * kFewOutputs;
    if (n0 >= a.N) return;
    const Row xrow = row_of(a.a, 0, 0x7fffffffu), wrow = row_of(a.w, n0 * K, 0x7fffffffu);
    const int r = lane & 15;
    const uint32_t xo = static_cast<uint32_t>(held(r, last_of(a.M, 0, kFewOutputs))) * K + (lane >> 4) * 16;
    const uint32_t wo = static_cast<uint32_t>(held(r, last_of(a.N, n0, kFewOutputs))) * K + (lane >> 4) * 16;

    Sum acc = mac::zero();
    auto multiply = [&](const i32x4 (&x)[2], const i32x4 (&w)[2]) __attribute__((always_inline)) {
        const typename mac::Frag xf = mac::frag(x[0], x[1]), wf = mac::frag(w[0], w[1]);
#pragma unroll
        for (int h = 0; h < mac::kParts; ++h) acc = mac::add(wf, xf, acc, h);
    };
    // kFewDepth steps are requested before the first of them is multiplied; steps beyond the whole ones are read again and not used
    for (int t = wave; t < whole; t += kFewDepth * kFewWaves) {
        i32x4 x[kFewDepth][2], w[kFewDepth][2];
#pragma unroll
        for (int d = 0; d < kFewDepth; ++d) {
            const int k0 = (t + d * kFewWaves < whole ? t + d * kFewWaves : t) * kBlockK;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                w[d][h] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(wrow, wo + 64 * h, k0, 0));
                x[d][h] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(xrow, xo + 64 * h, k0, 0));
            }
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int d = 0; d < kFewDepth; ++d)
            if (t + d * kFewWaves < whole) multiply(x[d], w[d]);
    }
    if (K % kBlockK != 0 && wave == whole % kFewWaves) {
        i32x4 x[2], w[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int left = K - whole * kBlockK - (lane >> 4) * 16 - 64 * h;
            w[h] = __builtin_bit_cast(i32x4, load_codes16(wrow, wo + 64 * h, whole * kBlockK, left));
            x[h] = __builtin_bit_cast(i32x4, load_codes16(xrow, xo + 64 * h, whole * kBlockK, left));
        }
        multiply(x, w);
    }

    part[wave][lane] = acc;
    __syncthreads();
    // lane l: row l % 16 of a, features 4 (l / 16) .. + 3
    for (int o = threadIdx.x; o < kFewOutputs * kFewOutputs; o += kFewWaves * kWave) {
        const int m = o / kFewOutputs, f = o % kFewOutputs;
        const int64_t n = n0 + f;
        if (m >= a.M || n >= a.N) continue;
        const int l = f / 4 * 16 + m, e = f % 4;
        auto sum = part[0][l][e];
#pragma unroll
        for (int w = 1; w < kFewWaves; ++w) sum += part[w][l][e];
        const float sa = a.sa[m], sw = a.sw[n];
        float v = static_cast<float>(sum) * sa * sw;
        if (!plain_scale(sa)) v = far_scaled(static_cast<float>(sum), sa, sw);
        if constexpr (std::is_same<Tag, bf16_io>::value) {
            if (a.bias) v += static_cast<float>(static_cast<const __bf16*>(a.bias)[n]);
            static_cast<__bf16*>(a.y)[m * a.N + n] = static_cast<__bf16>(v);
        } else {
            if (a.bias) v += static_cast<const float*>(a.bias)[n];
            static_cast<float*>(a.y)[m * a.N + n] = v;
        }
    }
}

// ---- large products ------------------------------------------------------------------------------------------------
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
//
// 32 760 x 5120 by 15 360, int8 to bf16: 128 x 128 tiles by four waves 4589 us, 256 x 256 2520, each operand brought while its waves
// multiply and w two steps ahead 2300, tiles in turn 2187, one sequence of steps and outputs past the caches 1980 to 2040: 2.55
// to 2.60e15 operations a second.  8190 x 5120 by 13 824 e4m3 436 us, 2.66e15.  The matrix units are busy 64 and 71 % of the
// time; a loop of such instructions alone reaches 81 % of their peak rate.
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
    meet();
    if (second) meet();
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
            meet();
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
            meet();
            at = at == 2 ? 0 : at + 1;
            odd ^= 1;
        };
#pragma unroll 1
        for (int t = 0; t < steps; ++t) step(t);
        store_products<C, Tag, TM, TN>(a, acc, m, n);
        if (!more) break;
        tile = next;
        here = there;
    }
    if (!second) meet();
}

}  // namespace lnmod
