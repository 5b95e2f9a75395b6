// lnmod_rotary.hpp -- arguments and host-side plan of the rotation and of the query and key norm with it.
#pragma once
#include "lnmod_launch.hpp"

namespace lnmod {

constexpr int kMaxAxes = 4;

// A tensor [B, S, heads, head_dim] whose features are dense: strides in bytes.
struct HeadsView {
    const char* p;
    int64_t batch, token, head;
};

struct RotaryPlan {
    const int32_t* positions;        // [S, axes], or [B*S, axes] with per_token
    const float* table;              // [table_rows, half, 2]: cosine and sine
    uint32_t table_rows;
    int32_t half;                    // pairs of a head
    int32_t axes;
    int32_t per_token;
    int32_t first[kMaxAxes];         // first pair of each axis
    int32_t part;                    // a head has features that are not turned
};

// One of the two tensors, and how its tokens and heads are shared out.
struct RotarySide {
    HeadsView x, dy;
    const void* w;
    float* rstd;                     // [N], or [N, heads] where each head has a norm
    void* y;                         // dense [N, heads, head_dim]: the result, or dx
    float* ws;                       // slots of `width` sums, one for each block
    int32_t heads, width;            // width: features of w
    float inv_width;
    int32_t hs_log2;                 // groups of lanes that take a token's heads
    int32_t waves, teams;            // waves of a token, tokens (or sets of neighbouring tokens) of a block
    int32_t chunks, chunk_heads;     // a token's heads in pieces for different blocks, where they are many and have no sum
    int32_t members, blocks;         // blocks = members * chunks
};

struct RotaryArgs {
    RotarySide side[2];
    RotaryPlan rot;
    int64_t N;                       // tokens of all samples
    int32_t S;
    int32_t head_dim, units, g_log2; // units of a head, lanes that a head takes
    float eps, sign;
    Divider sample_of;
};

struct RotaryDwArgs {
    const float* ws[2];
    void* dw[2];
    int32_t slots[2], width[2];
};

enum RotaryNorm { kNoNorm = 0, kRowNorm = 1, kHeadNorm = 2 };

struct RotaryShape {
    int vpl, block_waves, per_cu;    // units of a lane, waves of a block, blocks of a CU (both tensors together)
};

inline int ceil_log2(int64_t v) {
    int k = 0;
    while ((int64_t{1} << k) < v) ++k;
    return k;
}

// Heads that meet in a wave side by side, and rounds of them that a token's heads take.
struct HeadSplit {
    int hs_log2, rounds;
};
inline HeadSplit head_split(int heads, int g_log2) {
    const int most = 6 - g_log2, want = ceil_log2(heads);
    const int hs = want < most ? want : most;
    return {hs, (heads + (1 << hs) - 1) >> hs};
}

// Fills the shares of both tensors.
inline void plan_rotary(RotaryArgs& a, const RotaryShape& sh, bool chunked) {
    int64_t weight[2] = {0, 0};
    for (int t = 0; t < 2; ++t) {
        RotarySide& s = a.side[t];
        if (s.heads == 0) {
            s.chunks = s.waves = s.teams = 1;
            s.members = s.blocks = 0;
            continue;
        }
        const HeadSplit hp = head_split(s.heads, a.g_log2);
        s.hs_log2 = hp.hs_log2;
        int waves = (hp.rounds + sh.vpl - 1) / sh.vpl;
        s.chunks = 1;
        if (chunked && waves > sh.block_waves) {
            s.chunks = (waves + sh.block_waves - 1) / sh.block_waves;
            waves = (waves + s.chunks - 1) / s.chunks;
        }
        s.waves = waves;
        s.chunk_heads = (waves * sh.vpl) << hp.hs_log2;
        s.teams = sh.block_waves / waves;
        weight[t] = s.heads;
    }
    for (int t = 0; t < 2; ++t) {
        RotarySide& s = a.side[t];
        if (s.heads == 0) continue;
        const int64_t tokens = static_cast<int64_t>(s.teams) << (6 - a.g_log2 - s.hs_log2);
        const int64_t need = (a.N + tokens - 1) / tokens;
        int64_t most = static_cast<int64_t>(kNumCU) * sh.per_cu * weight[t] / ((weight[0] + weight[1]) * s.chunks);
        if (most < 1) most = 1;
        s.members = static_cast<int32_t>(need < most ? need : most);
        s.blocks = s.members * s.chunks;
    }
}

// slots of partial weight gradients of q and of k
void rotary_bwd_slots(int dtype, int64_t N, const int32_t (&heads)[2], int head_dim, int norm, int64_t (&slots)[2]);

hipError_t launch_rotary_fwd(int dtype, int norm, bool halves, RotaryArgs a, hipStream_t st);
hipError_t launch_rotary_bwd(int dtype, int norm, bool halves, RotaryArgs a, void* const (&dw)[2], bool io_grads, float* ws,
                             hipStream_t st);

}  // namespace lnmod
