// lnmod_rowcodes_kernels.hpp -- gfx950 device code of codes with one scale for a row (lnmod_code.hpp has the codes).
//
// A row stays in registers between its maximum and its codes, so it is read once: 2^lanes_log2 lanes hold a short row, K waves
// a long one.  Rows beyond what sixteen waves hold are read twice, the second time from the caches.
//
// HBM bounds it: 32 760 x 5120 bf16 to e4m3 88 us, 5.7 TB/s; 1025 x 13 824 9.3 us, 4.5 TB/s, with 7 us in the bytes.  Rows of 65 to 192
// units have two of them a lane, longer ones four (lnmod_rowcodes.hip).
#pragma once
#include "lnmod_code.hpp"

namespace lnmod {

struct RowCodesArgs {
    const void* x;
    void* codes;
    float* scales;
    int64_t N;
    int32_t D;
    int32_t units;           // D / 8
    int32_t lanes_log2;      // of a row, where a wave holds several (waves 1)
    int32_t waves;           // of a row
    int32_t keep;            // see keep_codes
};

// Largest of 2^bits neighbouring lanes (bits uniform); every one of them returns it.
__device__ inline uint32_t lanes_max(uint32_t v, int bits) {
    v = dpp_max<0xB1>(v, bits > 0 ? ~0u : 0u);
    v = dpp_max<0x4E>(v, bits > 1 ? ~0u : 0u);
    v = dpp_max<0x141>(v, bits > 2 ? ~0u : 0u);
    v = dpp_max<0x140>(v, bits > 3 ? ~0u : 0u);
    if (bits > 4) {
        const uint32_t t = __shfl_xor(v, 16);
        v = t > v ? t : v;
    }
    if (bits > 5) {
        const uint32_t t = __shfl_xor(v, 32);
        v = t > v ? t : v;
    }
    return v;
}

constexpr int kRowCodesWaves = 16;           // most waves of a block

template <typename Tag, typename C, int VPL>
__global__ __launch_bounds__(kRowCodesWaves* kWave) void row_codes_kernel(const RowCodesArgs a) {
    using unit = Unit<Tag>;
    __shared__ uint32_t most[2][kRowCodesWaves];
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int team = wave / a.waves, part = wave - team * a.waves, teams = (blockDim.x / kWave) / a.waves;
    const int u = lane & ((1 << a.lanes_log2) - 1);
    const int rows_log2 = 6 - a.lanes_log2;                       // rows of a wave
    const int64_t stride = (static_cast<int64_t>(gridDim.x) * teams) << rows_log2;
    int buf = 0;
    for (int64_t first = (static_cast<int64_t>(blockIdx.x) * teams) << rows_log2; first < a.N; first += stride) {
        const int64_t row = first + (static_cast<int64_t>(team) << rows_log2) + (lane >> a.lanes_log2);
        const bool here = row < a.N;
        const char* x = static_cast<const char*>(a.x) + (here ? row : a.N - 1) * static_cast<int64_t>(a.units) * unit::kBytes;
        u32x4 q[VPL][unit::NV];
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            const int c = ((i * a.waves + part) << a.lanes_log2) + u;
            const int cc = c < a.units ? c : a.units - 1;          // a feature that counts already
#pragma unroll
            for (int h = 0; h < unit::NV; ++h)
                q[i][h] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(x + static_cast<int64_t>(cc) * unit::kBytes) + h);
        }
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            const uint32_t t = unit::amax_bits(q[i]);
            m = t > m ? t : m;
        }
        m = lanes_max(m, a.lanes_log2);
        if (a.waves > 1) {
            if (lane == 0) most[buf][wave] = m;
            __syncthreads();
            for (int w = 0; w < a.waves; ++w) {
                const uint32_t t = most[buf][team * a.waves + w];
                m = t > m ? t : m;
            }
            buf ^= 1;
        }
        const Scale sc = scale_of<C>(m);
        if (here && u == 0 && part == 0) a.scales[row] = sc.s;
        char* codes = static_cast<char*>(a.codes) + row * a.D;
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            const int c = ((i * a.waves + part) << a.lanes_log2) + u;
            if (!here || c >= a.units) continue;
            float v[8];
            unit::unpack(q[i], v);
            u32x2* to = reinterpret_cast<u32x2*>(codes + static_cast<int64_t>(c) * 8);
            if (a.keep) *to = encode<C>(v, sc);
            else __builtin_nontemporal_store(encode<C>(v, sc), to);
        }
    }
}

// A row of any length by one block.
template <typename Tag, typename C>
__global__ __launch_bounds__(kRowCodesWaves* kWave) void long_row_codes_kernel(const RowCodesArgs a) {
    using unit = Unit<Tag>;
    __shared__ uint32_t most[2][kRowCodesWaves];
    const int wave = threadIdx.x >> 6;
    int buf = 0;
    for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
        const u32x4* x = reinterpret_cast<const u32x4*>(static_cast<const char*>(a.x) + row * static_cast<int64_t>(a.units) * unit::kBytes);
        uint32_t m = 0;
        for (int c = threadIdx.x; c < a.units; c += blockDim.x) {
            u32x4 q[unit::NV];
#pragma unroll
            for (int h = 0; h < unit::NV; ++h) q[h] = x[static_cast<int64_t>(c) * unit::NV + h];
            const uint32_t t = unit::amax_bits(q);
            m = t > m ? t : m;
        }
        m = lanes_max(m, 6);
        if ((threadIdx.x & (kWave - 1)) == 0) most[buf][wave] = m;
        __syncthreads();
        for (int w = 0; w < kRowCodesWaves; ++w) {
            const uint32_t t = most[buf][w];
            m = t > m ? t : m;
        }
        buf ^= 1;
        const Scale sc = scale_of<C>(m);
        if (threadIdx.x == 0) a.scales[row] = sc.s;
        u32x2* codes = reinterpret_cast<u32x2*>(static_cast<char*>(a.codes) + row * a.D);
        for (int c = threadIdx.x; c < a.units; c += blockDim.x) {
            u32x4 q[unit::NV];
#pragma unroll
            for (int h = 0; h < unit::NV; ++h) q[h] = x[static_cast<int64_t>(c) * unit::NV + h];
            float v[8];
            unit::unpack(q, v);
            codes[c] = encode<C>(v, sc);
        }
    }
}

}  // namespace lnmod
