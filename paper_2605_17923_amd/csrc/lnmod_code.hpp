// lnmod_code.hpp -- gfx950 device code shared by the kernels that hold activations in 8 bits: rows in units of eight
// features per lane, codes of a group of features with one scale, and the way back.
//
//   amax = max |v| of the group    s = fp32(max(amax, 2^-100) / Q)    r = fp32(1 / s)    Q = 127 (int8), 448 (e4m3)
//   int8: code = v*r to the nearest whole number, ties to even, in one rounding
//   e4m3: code = v*r rounded to fp32, then to the nearest e4m3, ties to even
//   the code stands for code*s.  A group that holds an infinity or a NaN has s = NaN and the codes 0.
//
// The codes are a function of the group's values alone, bit for bit: both quotients are correctly rounded, so any
// program that follows these lines gets the same codes.  |v*r| stays below Q (1 + 2^-21), which rounds to Q.  The floor
// of 2^-100 keeps s and r normal numbers; a group of zeros has the codes 0.
#pragma once
#include "lnmod_code_shapes.hpp"
#include "lnmod_kernels.hpp"

namespace lnmod {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

constexpr int kUnit = 8;                     // features per lane and chunk, in either element type
constexpr int kDepth = 2;                    // steps of rows in registers: the one that is computed and the one requested

// ---- eight features of a row in one lane ------------------------------------------------------------------------
template <typename Tag> struct Unit;

template <> struct Unit<bf16_io> {
    static constexpr int NV = 1;             // 16-byte vectors
    static constexpr uint32_t kBytes = 16;
    __device__ static inline void unpack(const u32x4 (&q)[1], float (&v)[8]) { IO<bf16_io>::unpack(q[0], v); }
    __device__ static inline void pack(const float (&v)[8], u32x4 (&q)[1]) { q[0] = IO<bf16_io>::pack(v); }
    // bits of the largest |v| as fp32, NaN above infinity above every number
    __device__ static inline uint32_t amax_bits(const u32x4 (&q)[1]) {
        u16x2 m = __builtin_bit_cast(u16x2, q[0][0] & 0x7fff7fffu);
#pragma unroll
        for (int j = 1; j < 4; ++j) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, q[0][j] & 0x7fff7fffu));
        const uint32_t b = __builtin_bit_cast(uint32_t, m);
        const uint32_t lo = b << 16, hi = b & 0xffff0000u;
        return lo > hi ? lo : hi;
    }
};

template <> struct Unit<f32_io> {
    static constexpr int NV = 2;
    static constexpr uint32_t kBytes = 32;
    __device__ static inline void unpack(const u32x4 (&q)[2], float (&v)[8]) {
        const f32x4 a = __builtin_bit_cast(f32x4, q[0]), b = __builtin_bit_cast(f32x4, q[1]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = a[j];
            v[4 + j] = b[j];
        }
    }
    __device__ static inline void pack(const float (&v)[8], u32x4 (&q)[2]) {
        const f32x4 a = {v[0], v[1], v[2], v[3]}, b = {v[4], v[5], v[6], v[7]};
        q[0] = __builtin_bit_cast(u32x4, a);
        q[1] = __builtin_bit_cast(u32x4, b);
    }
    __device__ static inline uint32_t amax_bits(const u32x4 (&q)[2]) {
        uint32_t m = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t b = q[h][j] & 0x7fffffffu;
                m = b > m ? b : m;
            }
        }
        return m;
    }
};

// A row as a buffer of its own: a read beyond its end gives zeros and a write beyond it does nothing, so lanes without
// features, and rows beyond the last one (0 bytes), need no branch and no address of their own.  With a comparison and an
// execution mask around every access the forward's loop was cut into thirty blocks, and a 64-bit address was formed for each.
typedef __amdgpu_buffer_rsrc_t Row;
constexpr uint32_t kNowhere = 0x7ffffff0u;   // an offset beyond every row
constexpr int kStream = 2;                   // cache policy: nontemporal

__device__ inline Row row_of(const void* base, int64_t uniform_off, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(base)) + uniform64(uniform_off), 0,
                                             static_cast<int>(bytes), 0x00027000);
}
template <typename Tag, int POLICY = kStream>
__device__ inline void load_unit(Row row, uint32_t chunk, u32x4 (&q)[Unit<Tag>::NV]) {
#pragma unroll
    for (int h = 0; h < Unit<Tag>::NV; ++h)
        q[h] = __builtin_amdgcn_raw_buffer_load_b128(row, static_cast<int>(chunk * Unit<Tag>::kBytes + 16u * h), 0, POLICY);
}
template <typename Tag>
__device__ inline void store_unit(Row row, uint32_t chunk, const u32x4 (&q)[Unit<Tag>::NV]) {
#pragma unroll
    for (int h = 0; h < Unit<Tag>::NV; ++h)
        __builtin_amdgcn_raw_buffer_store_b128(q[h], row, static_cast<int>(chunk * Unit<Tag>::kBytes + 16u * h), 0, kStream);
}
// Eight codes are eight bytes of a lane.
__device__ inline u32x2 load_codes(Row row, uint32_t chunk) {
    return __builtin_amdgcn_raw_buffer_load_b64(row, static_cast<int>(chunk * 8u), 0, kStream);
}
// keep (uniform): codes that the last-level cache can hold stay there for their reader, see keep_codes.
__device__ inline void store_codes(Row row, uint32_t chunk, const u32x2& c, int32_t keep) {
    if (keep) __builtin_amdgcn_raw_buffer_store_b64(c, row, static_cast<int>(chunk * 8u), 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b64(c, row, static_cast<int>(chunk * 8u), 0, kStream);
}
// One float of a row; the scales of a row are shared by the waves of a block, so they stay in the cache.
__device__ inline float load_float(Row row, uint32_t offset) {
    return __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(row, static_cast<int>(offset), 0, 0));
}
__device__ inline void store_float(Row row, uint32_t offset, float v) {
    __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v), row, static_cast<int>(offset), 0, 0);
}
// Eight partial sums of a lane; they stay in the cache for the second pass.
__device__ inline void store_sums8(Row row, uint32_t chunk, const float (&v)[8]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const f32x4 t = {v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, t), row, static_cast<int>(chunk * 32u + 16u * h), 0, 0);
    }
}
// ---- several rows in a block -----------------------------------------------------------------------------------------------
// Where one wave holds a row, the waves of a block take rows of their own, and what they have summed meets in LDS at the end: a
// slot of partial sums per block in place of one per wave, and blocks that the dispatcher spreads over the CUs evenly.  The
// waves are added in their order.
constexpr int fwd_groups_most(int k) { return k > 1 ? 1 : kFwdGroups; }
constexpr int groups_most(int k, int waves_per_simd) { return k > 1 ? 1 : 4 * waves_per_simd; }
// units of a lane that meet at a time, so that LDS stays below the 64 KB that a block gets without asking
constexpr int units_at_once(int vpl, int waves_per_simd) {
    const int most = waves_per_simd == 1 ? 4 : waves_per_simd == 2 ? 2 : 1;
    return vpl < most ? vpl : most;
}
constexpr size_t group_lds(int groups, int units, int sums) { return static_cast<size_t>(groups - 1) * units * sums * kWave * kUnit * 4; }

// acc[..][i] of the waves beyond the first one are added to the first one's; every wave of the block calls it.
template <int UNITS, int VPL, int SUMS>
__device__ inline void add_groups(float (&acc)[SUMS][VPL][8], int group, int groups, f32x4* lds) {
    if (groups == 1) return;
    const int lane = threadIdx.x & (kWave - 1);
    constexpr int kHalves = SUMS * UNITS * 2;
#pragma unroll
    for (int i0 = 0; i0 < VPL; i0 += UNITS) {
        if (group > 0) {
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
                const int i = i0 + h / 2 % UNITS, e = h % 2 * 4;
                if (i >= VPL) continue;
                const float(&v)[8] = acc[h / (UNITS * 2)][i];
                lds[((group - 1) * kHalves + h) * kWave + lane] = f32x4{v[e], v[e + 1], v[e + 2], v[e + 3]};
            }
        }
        __syncthreads();
        if (group == 0) {
            for (int g = 0; g < groups - 1; ++g) {
#pragma unroll
                for (int h = 0; h < kHalves; ++h) {
                    const int i = i0 + h / 2 % UNITS;
                    if (i >= VPL) continue;
                    const f32x4 t = lds[(g * kHalves + h) * kWave + lane];
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[h / (UNITS * 2)][i][h % 2 * 4 + e] += t[e];
                }
            }
        }
        __syncthreads();                                     // before the next sums
    }
}

// A float that no kernel of the launch writes, at a uniform address: a scalar load (see table_at).
typedef const float __attribute__((address_space(4))) * const_f32_ptr;
__device__ inline float float_at(const float* p, int64_t i) { return ((const_f32_ptr)p)[i]; }

template <int NV>
__device__ inline void opaque(u32x4 (&q)[NV]) {        // the fp32 values are rebuilt behind this, not carried across it
#pragma unroll
    for (int h = 0; h < NV; ++h) asm volatile("" : "+v"(q[h]));
}

// ---- largest magnitude of a group: 4, 8 or 16 consecutive lanes, inside one DPP row ----------------------------------
template <int CTRL> __device__ inline uint32_t dpp_max(uint32_t v, uint32_t mask = ~0u) {
    const uint32_t t = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, 0xf, 0xf, false)) & mask;
    return t > v ? t : v;
}
// Every lane of the group returns it; all 64 lanes take part.  lanes_log2 is uniform: 2, 3 or 4; the steps that a smaller
// group has none of are masked, not branched around.
__device__ inline uint32_t group_max(uint32_t v, int lanes_log2) {
    v = dpp_max<0xB1>(v);                                     // quad_perm [1,0,3,2]
    v = dpp_max<0x4E>(v);                                     // quad_perm [2,3,0,1]
    v = dpp_max<0x141>(v, lanes_log2 > 2 ? ~0u : 0u);         // row_half_mirror
    return dpp_max<0x140>(v, lanes_log2 > 3 ? ~0u : 0u);      // row_mirror
}
__device__ inline uint32_t row16_max(uint32_t v) { return group_max(v, 4); }

// ---- codes ------------------------------------------------------------------------------------------------------
struct int8_code {
    static constexpr float kLargest = 127.0f;
};
struct e4m3_code {
    static constexpr float kLargest = 448.0f;
};

struct Scale {
    float s, r;                              // both NaN where the group holds an infinity or a NaN
    bool good;
};

// s and r of a group.  A division costs a dozen instructions; these two are a product, a reciprocal and four fused steps:
// with c = fp32(1/Q), q = a*c and the exact remainder a - Q q, q + c (a - Q q) is the correctly rounded a / Q (Markstein's
// theorem on division by fused multiply-add; for Q = 127 and 448 checked for every significand of a), and one Newton step on
// the hardware's reciprocal gives the correctly rounded 1 / s (checked for every significand of s).  An infinity leaves
// a - Q q without a value, so s is NaN without being asked for.
template <typename C>
__device__ inline Scale scale_of(uint32_t amax_bits) {
    constexpr float Q = C::kLargest, c = 1.0f / Q;
    constexpr uint32_t kFloor = 0x0d800000u;                 // 2^-100
    const float a = __builtin_bit_cast(float, amax_bits > kFloor ? amax_bits : kFloor);
    const float q = a * c;
    const float s = __builtin_fmaf(__builtin_fmaf(-Q, q, a), c, q);
    float r = __builtin_amdgcn_rcpf(s);
    r = __builtin_fmaf(__builtin_fmaf(-s, r, 1.0f), r, r);
    return Scale{s, r, amax_bits < 0x7f800000u};
}

template <typename C> __device__ u32x2 encode(const float (&v)[8], const Scale& sc);

// 1.5 * 2^23 + code: the fused sum rounds v*r once, and the low byte of its bits is the code
template <>
__device__ inline u32x2 encode<int8_code>(const float (&v)[8], const Scale& sc) {
    u32x2 w;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t t[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) t[j] = __builtin_bit_cast(uint32_t, __builtin_fmaf(v[4 * h + j], sc.r, 0x1.8p23f));
        const uint32_t lo = __builtin_amdgcn_perm(t[1], t[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(t[3], t[2], 0x04000c0cu);
        w[h] = sc.good ? lo | hi : 0u;
    }
    return w;
}

template <>
__device__ inline u32x2 encode<e4m3_code>(const float (&v)[8], const Scale& sc) {
    u32x2 w;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        int t = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h] * sc.r, v[4 * h + 1] * sc.r, 0, false);
        t = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h + 2] * sc.r, v[4 * h + 3] * sc.r, t, true);
        w[h] = sc.good ? static_cast<uint32_t>(t) : 0u;
    }
    return w;
}

// The numbers that eight codes are, not yet times the scale.
template <typename C> __device__ void decode(const u32x2& w, float (&v)[8]);

template <>
__device__ inline void decode<int8_code>(const u32x2& w, float (&v)[8]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int t = static_cast<int>(w[h]);
        v[4 * h] = static_cast<float>(static_cast<int8_t>(t));
        v[4 * h + 1] = static_cast<float>(static_cast<int8_t>(t >> 8));
        v[4 * h + 2] = static_cast<float>(static_cast<int8_t>(t >> 16));
        v[4 * h + 3] = static_cast<float>(t >> 24);
    }
}

template <>
__device__ inline void decode<e4m3_code>(const u32x2& w, float (&v)[8]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[h]), false);
        const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[h]), true);
        v[4 * h] = a[0];
        v[4 * h + 1] = a[1];
        v[4 * h + 2] = b[0];
        v[4 * h + 3] = b[1];
    }
}

// What eight codes stand for.  The largest float has s = fp32(max / 127) rounded up, and 127*s is beyond float32 (no other
// largest value of a group does that, and none in e4m3, 448 = 7 * 2^6 and max = 7 * 2396745 * 2^104): such a product is held
// to the largest float, so that a finite group, a mask of the type's lowest value among them, stays finite.  Rounded to bf16 it is the
// infinity that max itself rounds to.  One instruction per feature of fp32 int8: 20 000 x 5120 back 97.9 -> 100.5 us.
template <typename Tag, typename C>
__device__ inline void stand_for(const u32x2& w, float s, float (&v)[8]) {
    decode<C>(w, v);
    // with two NaN beside it the median is v itself
    [[maybe_unused]] const float most = __builtin_fabsf(s) < __builtin_inff() ? __FLT_MAX__ : __builtin_nanf("");
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        v[e] *= s;
        if constexpr (std::is_same<Tag, f32_io>::value && std::is_same<C, int8_code>::value)
            v[e] = __builtin_amdgcn_fmed3f(v[e], -most, most);
    }
}

}  // namespace lnmod
