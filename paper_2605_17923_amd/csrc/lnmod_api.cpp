// lnmod_api.cpp -- the C ABI declared in include/lnmod.h: the operator entry points, nothing else.
// The library keeps no mutable state: a call's result depends on its arguments alone.
#include "lnmod_api_impl.hpp"

static_assert(LNMOD_STATIC_WORKSPACE_BYTES == lnmod::kStaticWorkspaceBytes, "header and library disagree");

namespace {

using lnmod::Problem;
using namespace lnmod::api;

size_t gated_workspace_bytes(int64_t nseg, int64_t T, int64_t D) {
    int64_t slots = 0;
    for (int dtype = 0; dtype < 2; ++dtype) {
        if (D % (dtype == 0 ? 8 : 4) != 0) continue;
        const lnmod::RowPlan pl = lnmod::gated_bwd_plan(T, nseg, D, dtype);
        const int64_t s = lnmod::bwd_slots(pl, nseg);
        if (s > slots) slots = s;
    }
    return static_cast<size_t>(slots) * 3u * static_cast<size_t>(D) * sizeof(float);
}

size_t qknorm_workspace_bytes(int64_t N, int64_t D) {
    int64_t nb = 0;
    for (int dtype = 0; dtype < 2; ++dtype) {
        if (D % (dtype == 0 ? 8 : 4) != 0) continue;
        const int64_t b = lnmod::qknorm_bwd_blocks(N, D, dtype);
        if (b > nb) nb = b;
    }
    return static_cast<size_t>(2 * nb) * static_cast<size_t>(D) * sizeof(float);
}

// (segments, tokens per sample, total tokens) of a gated call, or false on overflow
bool gated_shape(const int32_t* cu, int64_t B_or_nseg, int64_t S_or_T, int64_t* S, int64_t* T) {
    if (cu) {
        *S = 0;
        *T = S_or_T;
        return true;
    }
    *S = S_or_T;
    *T = total_tokens(B_or_nseg, S_or_T);
    return *T >= 0;
}

int gated_backward_impl(const void* dy, const void* dh, const void* h, const void* u,
                         const void* gate, const void* scale, const int32_t* cu_seqlens,
                         int64_t B_or_nseg, int64_t S_or_T, int64_t D, float eps, void* stream,
                         const float* mean, const float* rstd, void* dx, void* du, void* dgate,
                         void* dshift, void* dscale, void* workspace, size_t workspace_size,
                         int dtype, bool io_grads) {
    int64_t S, T;
    if (!gated_shape(cu_seqlens, B_or_nseg, S_or_T, &S, &T)) return LNMOD_EINVAL;
    const int st = check_shape(B_or_nseg, S_or_T, D, eps, dtype, T);
    if (st != LNMOD_OK) return st;
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    if (T == 0) {
        if (B_or_nseg > 0) {                                  // empty sums are zeros
            if (!dgate || !dshift || !dscale) return LNMOD_EINVAL;
            if (io_grads && (!aligned16(dgate) || !aligned16(dshift) || !aligned16(dscale))) return LNMOD_EALIGN;
            const auto zero = [&](void* p) {
                return lnmod::launch_zero_f32(static_cast<float*>(p), grad_floats(B_or_nseg * D, dtype, io_grads), hs);
            };
            hipError_t e = zero(dgate);
            if (e == hipSuccess) e = zero(dshift);
            if (e == hipSuccess) e = zero(dscale);
            return e == hipSuccess ? LNMOD_OK : LNMOD_ELAUNCH;
        }
        return LNMOD_OK;
    }
    if (B_or_nseg == 0) return LNMOD_EINVAL;
    if (!dy || !dh || !h || !u || !gate || !scale || !mean || !rstd || !dx || !du || !dgate ||
        !dshift || !dscale)
        return LNMOD_EINVAL;
    if (!aligned16(dy) || !aligned16(dh) || !aligned16(h) || !aligned16(u) || !aligned16(gate) ||
        !aligned16(scale) || !aligned16(dx) || !aligned16(du) || !aligned16(dgate) ||
        !aligned16(dshift) || !aligned16(dscale))
        return LNMOD_EALIGN;
    if (!workspace || workspace_size < gated_workspace_bytes(B_or_nseg, T, D)) return LNMOD_EWORKSPACE;
    if (!aligned16(workspace)) return LNMOD_EALIGN;
    const Problem p{dtype, cu_seqlens, B_or_nseg, S, T, D, eps};
    const hipError_t e = lnmod::launch_gated_bwd(p, dy, dh, h, u, gate, scale, mean, rstd, dx, du,
                                                 dgate, dshift, dscale, io_grads,
                                                 static_cast<float*>(workspace), hs);
    return e == hipSuccess ? LNMOD_OK : LNMOD_ELAUNCH;
}

int qknorm_backward_impl(const void* dq_out, const void* dk_out, const void* q, const void* k,
                          const void* wq, const void* wk, int64_t N, int64_t D, float eps,
                          void* stream, const float* rstd_q, const float* rstd_k, void* dq, void* dk,
                          void* dwq, void* dwk, void* workspace, size_t workspace_size, int dtype, bool io_grads) {
    const int st = check_shape(1, N, D, eps, dtype, N);
    if (st != LNMOD_OK) return st;
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    if (N == 0) {                                             // empty sums are zeros
        if (!dwq || !dwk) return LNMOD_EINVAL;
        if (io_grads && (!aligned16(dwq) || !aligned16(dwk))) return LNMOD_EALIGN;
        const auto zero = [&](void* p) {
            return lnmod::launch_zero_f32(static_cast<float*>(p), grad_floats(D, dtype, io_grads), hs);
        };
        hipError_t e = zero(dwq);
        if (e == hipSuccess) e = zero(dwk);
        return e == hipSuccess ? LNMOD_OK : LNMOD_ELAUNCH;
    }
    if (!dq_out || !dk_out || !q || !k || !wq || !wk || !rstd_q || !rstd_k || !dq || !dk || !dwq || !dwk)
        return LNMOD_EINVAL;
    if (!aligned16(dq_out) || !aligned16(dk_out) || !aligned16(q) || !aligned16(k) || !aligned16(wq) ||
        !aligned16(wk) || !aligned16(dq) || !aligned16(dk) ||
        (io_grads && (!aligned16(dwq) || !aligned16(dwk))))
        return LNMOD_EALIGN;
    if (!workspace || workspace_size < qknorm_workspace_bytes(N, D)) return LNMOD_EWORKSPACE;
    if (!aligned16(workspace)) return LNMOD_EALIGN;
    const hipError_t e = lnmod::launch_qknorm_bwd(dtype, dq_out, dk_out, q, k, wq, wk, N, D, rstd_q,
                                                  rstd_k, dq, dk, dwq, dwk, io_grads,
                                                  static_cast<float*>(workspace), hs);
    return e == hipSuccess ? LNMOD_OK : LNMOD_ELAUNCH;
}

// ---- activations in 8 bits -------------------------------------------------------------------------------------
bool valid_group(int64_t group) { return group == 32 || group == 64 || group == 128; }
bool valid_code(int code) { return code == LNMOD_INT8 || code == LNMOD_E4M3; }

int check_rows(int64_t N, int64_t D, int64_t group, int dtype, int code) {
    if (N < 0 || N >= (int64_t(1) << 31) || D < 0 || !valid_group(group) || !valid_code(code)) return LNMOD_EINVAL;
    if (dtype != LNMOD_BF16 && dtype != LNMOD_F32) return LNMOD_EINVAL;
    if (D < 8 || D > (int64_t(1) << 20) || D % 8 != 0) return LNMOD_EUNSUPPORTED;
    return LNMOD_OK;
}

// For one sample a bound on the plan's slots that does not fall as the rows grow.
size_t ckpt_workspace_bytes(int64_t nseg, int64_t T, int64_t D) {
    int64_t slots = 0;
    for (int dtype = 0; dtype < 2; ++dtype) {
        const int64_t s = nseg == 1 ? lnmod::ckpt_bwd_most_slots(T, D, dtype)
                                    : lnmod::bwd_slots(lnmod::ckpt_bwd_plan(T, nseg, D, dtype), nseg);
        if (s > slots) slots = s;
    }
    return static_cast<size_t>(slots) * 2u * static_cast<size_t>(D) * sizeof(float);
}

size_t rmsq_workspace_bytes(int64_t N, int64_t D) {
    int64_t slots = 0;
    for (int dtype = 0; dtype < 2; ++dtype) {
        const int64_t s = lnmod::rmsq_bwd_most_slots(N, D, dtype);
        if (s > slots) slots = s;
    }
    return static_cast<size_t>(slots) * static_cast<size_t>(D) * sizeof(float);
}

// dr: a second copy of dx, or null
int rmsnorm_quant_backward_impl(const void* dy, const void* dh, const void* h, const void* w, int64_t N, int64_t D, void* stream,
                                const float* rstd, void* dx, void* dr, void* dw, void* workspace, size_t workspace_size,
                                int dtype, int io_grads) {
    const int st = check_shape(1, N, D, 1.0f, dtype, N);
    if (st != LNMOD_OK) return st;
    if (D % 8 != 0) return LNMOD_EUNSUPPORTED;
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    if (!dw) return LNMOD_EINVAL;
    if (io_grads && !aligned16(dw)) return LNMOD_EALIGN;
    if (N == 0) {                                                  // empty sums are zeros
        const hipError_t e = lnmod::launch_zero_f32(static_cast<float*>(dw), grad_floats(D, dtype, io_grads != 0), hs);
        return e == hipSuccess ? LNMOD_OK : LNMOD_ELAUNCH;
    }
    if (!dy || !h || !w || !rstd || !dx) return LNMOD_EINVAL;
    if (!aligned16(dy) || !aligned16(dh) || !aligned16(h) || !aligned16(w) || !aligned16(dx) || !aligned16(dr))
        return LNMOD_EALIGN;
    if (!workspace || workspace_size < rmsq_workspace_bytes(N, D)) return LNMOD_EWORKSPACE;
    if (!aligned16(workspace)) return LNMOD_EALIGN;
    const hipError_t e = lnmod::launch_rmsq_bwd(dtype, dy, dh, h, w, N, D, rstd, dx, dr, dw, io_grads != 0,
                                                static_cast<float*>(workspace), hs);
    return e == hipSuccess ? LNMOD_OK : LNMOD_ELAUNCH;
}

}  // namespace

extern "C" {

int lnmod_forward(const void* x, const void* shift, const void* scale, int64_t B, int64_t S,
                  int64_t D, float eps, void* stream, void* y, float* mean, float* rstd,
                  int dtype, int mod) {
    const int64_t T = total_tokens(B, S);
    if (T < 0) return LNMOD_EINVAL;
    return forward_impl(x, shift, scale, nullptr, false, B, S, T, D, eps, stream, y, mean, rstd,
                        dtype, mod);
}

int lnmod_backward(const void* dy, const void* x, const void* shift, const void* scale, int64_t B,
                   int64_t S, int64_t D, float eps, void* stream, const float* mean,
                   const float* rstd, void* dx, void* dshift, void* dscale, void* workspace,
                   size_t workspace_size, int dtype, int mod) {
    (void)shift;
    const int64_t T = total_tokens(B, S);
    if (T < 0) return LNMOD_EINVAL;
    return backward_impl(dy, x, scale, nullptr, false, B, S, T, D, eps, stream, mean, rstd, dx,
                         dshift, dscale, workspace, workspace_size, dtype, mod);
}

int lnmod_forward_varlen(const void* x, const void* shift, const void* scale,
                         const int32_t* cu_seqlens, int64_t nseg, int64_t T, int64_t D, float eps,
                         void* stream, void* y, float* mean, float* rstd, int dtype) {
    return forward_impl(x, shift, scale, cu_seqlens, true, nseg, 0, T, D, eps, stream, y, mean,
                        rstd, dtype, LNMOD_PER_SAMPLE);
}

int lnmod_backward_varlen(const void* dy, const void* x, const void* shift, const void* scale,
                          const int32_t* cu_seqlens, int64_t nseg, int64_t T, int64_t D, float eps,
                          void* stream, const float* mean, const float* rstd, void* dx,
                          void* dshift, void* dscale, void* workspace, size_t workspace_size,
                          int dtype) {
    (void)shift;
    return backward_impl(dy, x, scale, cu_seqlens, true, nseg, 0, T, D, eps, stream, mean, rstd,
                         dx, dshift, dscale, workspace, workspace_size, dtype, LNMOD_PER_SAMPLE);
}

int lnmod_backward_static(const void* dy, const void* x, const void* shift, const void* scale,
                          int64_t B, int64_t S, int64_t D, float eps, void* stream,
                          const float* mean, const float* rstd, void* dx, void* dshift,
                          void* dscale, int dtype, int mod) {
    (void)shift;
    const int64_t T = total_tokens(B, S);
    if (T < 0) return LNMOD_EINVAL;
    if (mod != LNMOD_PER_SAMPLE && mod != LNMOD_PER_TOKEN) return LNMOD_EINVAL;
    const int st = check_shape(B, S, D, eps, dtype, T);
    if (st != LNMOD_OK) return st;
    void* ws = nullptr;
    size_t ws_bytes = 0;
    lnmod::Shape shape{};
    const lnmod::Shape* force = nullptr;
    if (mod == LNMOD_PER_SAMPLE && T > 0 && B > 0) {
        // the slots of exactly this call's plan (element type and whether the statistics are
        // recomputed are known here), not the query's upper bound over all plans
        if ((mean == nullptr) != (rstd == nullptr)) return LNMOD_EINVAL;
        const int64_t max_slots = static_cast<int64_t>(lnmod::kStaticWorkspaceBytes / (2u * static_cast<size_t>(D) * sizeof(float)));
        if (!lnmod::bwd_shape_within(T, B, D, dtype, mean == nullptr, max_slots, &shape)) return LNMOD_EWORKSPACE;
        if (shape.clusters > 0) force = &shape;      // not the plan lnmod_backward takes: fewer slots
        // every other argument is checked before the first HIP call
        if (!dy || !x || !scale || !dx || !dshift || !dscale) return LNMOD_EINVAL;
        if (!aligned16(dy) || !aligned16(x) || !aligned16(scale) || !aligned16(dx) ||
            !aligned16(dshift) || !aligned16(dscale))
            return LNMOD_EALIGN;
        float* p = nullptr;
        if (lnmod::static_workspace(&p) != hipSuccess) return LNMOD_ELAUNCH;
        ws = p;
        ws_bytes = lnmod::kStaticWorkspaceBytes;
    }
    return backward_impl(dy, x, scale, nullptr, false, B, S, T, D, eps, stream, mean, rstd, dx,
                         dshift, dscale, ws, ws_bytes, dtype, mod, force, /*exact_workspace=*/true);
}

int lnmod_backward_io(const void* dy, const void* x, const void* scale, const int32_t* cu_seqlens,
                      int64_t B_or_nseg, int64_t S_or_T, int64_t D, float eps, void* stream,
                      const float* mean, const float* rstd, void* dx, void* dshift, void* dscale,
                      void* workspace, size_t workspace_size, int dtype) {
    int64_t S, T;
    if (!gated_shape(cu_seqlens, B_or_nseg, S_or_T, &S, &T)) return LNMOD_EINVAL;
    return backward_impl(dy, x, scale, cu_seqlens, cu_seqlens != nullptr, B_or_nseg, S, T, D, eps, stream, mean,
                         rstd, dx, dshift, dscale, workspace, workspace_size, dtype, LNMOD_PER_SAMPLE, nullptr,
                         false, /*io_grads=*/true);
}

int lnmod_backward_token(const void* dy, const void* x, const void* scale, int64_t B, int64_t S, int64_t D,
                         float eps, void* stream, const float* mean, const float* rstd, void* dx,
                         void* dscale, int dtype) {
    const int64_t T = total_tokens(B, S);
    if (T < 0) return LNMOD_EINVAL;
    return backward_impl(dy, x, scale, nullptr, false, B, S, T, D, eps, stream, mean, rstd, dx, nullptr, dscale,
                         nullptr, 0, dtype, LNMOD_PER_TOKEN, nullptr, false, false, /*no_dshift=*/true);
}

size_t lnmod_backward_workspace_bytes(int64_t B_or_nseg, int64_t total, int64_t D, int mod) {
    if (mod != LNMOD_PER_SAMPLE) return 0;
    if (B_or_nseg < 0 || total < 0 || total >= (int64_t(1) << 31)) return 0;
    if (D < 8 || D > lnmod::kMaxD || D % 4 != 0) return 0;
    return workspace_bytes(B_or_nseg, total, D);
}

const char* lnmod_status_string(int status) {
    switch (status) {
        case LNMOD_OK: return "ok";
        case LNMOD_EINVAL: return "invalid argument";
        case LNMOD_EUNSUPPORTED: return "unsupported hidden size or combination of arguments";
        case LNMOD_EALIGN: return "pointer not 16-byte aligned";
        case LNMOD_EWORKSPACE: return "workspace missing or too small";
        case LNMOD_ELAUNCH: return "kernel launch failed";
        default: return "unknown status";
    }
}

int lnmod_gated_forward(const void* x, const void* u, const void* gate, const void* shift,
                        const void* scale, const int32_t* cu_seqlens, int64_t B_or_nseg,
                        int64_t S_or_T, int64_t D, float eps, void* stream, void* h, void* y,
                        float* mean, float* rstd, int dtype) {
    int64_t S, T;
    if (!gated_shape(cu_seqlens, B_or_nseg, S_or_T, &S, &T)) return LNMOD_EINVAL;
    const int st = check_shape(B_or_nseg, S_or_T, D, eps, dtype, T);
    if (st != LNMOD_OK) return st;
    if (T == 0) return LNMOD_OK;
    if (B_or_nseg == 0) return LNMOD_EINVAL;
    if (!x || !u || !gate || !shift || !scale || !h || !y || !mean || !rstd) return LNMOD_EINVAL;
    if (!aligned16(x) || !aligned16(u) || !aligned16(gate) || !aligned16(shift) || !aligned16(scale) ||
        !aligned16(h) || !aligned16(y))
        return LNMOD_EALIGN;
    const Problem p{dtype, cu_seqlens, B_or_nseg, S, T, D, eps};
    const hipError_t e = lnmod::launch_gated_fwd(p, x, u, gate, shift, scale, h, y, mean, rstd,
                                                 static_cast<hipStream_t>(stream));
    return e == hipSuccess ? LNMOD_OK : LNMOD_ELAUNCH;
}

int lnmod_gated_backward(const void* dy, const void* dh, const void* h, const void* u,
                         const void* gate, const void* scale, const int32_t* cu_seqlens,
                         int64_t B_or_nseg, int64_t S_or_T, int64_t D, float eps, void* stream,
                         const float* mean, const float* rstd, void* dx, void* du, float* dgate,
                         float* dshift, float* dscale, void* workspace, size_t workspace_size,
                         int dtype) {
    return gated_backward_impl(dy, dh, h, u, gate, scale, cu_seqlens, B_or_nseg, S_or_T, D, eps, stream, mean, rstd,
                               dx, du, dgate, dshift, dscale, workspace, workspace_size, dtype, false);
}

int lnmod_gated_backward_io(const void* dy, const void* dh, const void* h, const void* u,
                            const void* gate, const void* scale, const int32_t* cu_seqlens,
                            int64_t B_or_nseg, int64_t S_or_T, int64_t D, float eps, void* stream,
                            const float* mean, const float* rstd, void* dx, void* du, void* dgate,
                            void* dshift, void* dscale, void* workspace, size_t workspace_size,
                            int dtype) {
    return gated_backward_impl(dy, dh, h, u, gate, scale, cu_seqlens, B_or_nseg, S_or_T, D, eps, stream, mean, rstd,
                               dx, du, dgate, dshift, dscale, workspace, workspace_size, dtype, true);
}

size_t lnmod_gated_backward_workspace_bytes(int64_t B_or_nseg, int64_t total, int64_t D) {
    if (B_or_nseg < 0 || total < 0 || total >= (int64_t(1) << 31)) return 0;
    if (D < 8 || D > lnmod::kMaxD || D % 4 != 0) return 0;
    return gated_workspace_bytes(B_or_nseg, total, D);
}

int lnmod_qknorm_forward(const void* q, const void* k, const void* wq, const void* wk, int64_t N,
                         int64_t D, float eps, void* stream, void* q_out, void* k_out,
                         float* rstd_q, float* rstd_k, int dtype) {
    const int st = check_shape(1, N, D, eps, dtype, N);
    if (st != LNMOD_OK) return st;
    if (N == 0) return LNMOD_OK;
    if (!q || !k || !wq || !wk || !q_out || !k_out || !rstd_q || !rstd_k) return LNMOD_EINVAL;
    if (!aligned16(q) || !aligned16(k) || !aligned16(wq) || !aligned16(wk) || !aligned16(q_out) ||
        !aligned16(k_out))
        return LNMOD_EALIGN;
    const hipError_t e = lnmod::launch_qknorm_fwd(dtype, q, k, wq, wk, N, D, eps, q_out, k_out, rstd_q,
                                                  rstd_k, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? LNMOD_OK : LNMOD_ELAUNCH;
}

int lnmod_qknorm_backward(const void* dq_out, const void* dk_out, const void* q, const void* k,
                          const void* wq, const void* wk, int64_t N, int64_t D, float eps,
                          void* stream, const float* rstd_q, const float* rstd_k, void* dq, void* dk,
                          float* dwq, float* dwk, void* workspace, size_t workspace_size, int dtype) {
    return qknorm_backward_impl(dq_out, dk_out, q, k, wq, wk, N, D, eps, stream, rstd_q, rstd_k, dq, dk, dwq, dwk,
                                workspace, workspace_size, dtype, false);
}

int lnmod_qknorm_backward_io(const void* dq_out, const void* dk_out, const void* q, const void* k,
                             const void* wq, const void* wk, int64_t N, int64_t D, float eps,
                             void* stream, const float* rstd_q, const float* rstd_k, void* dq, void* dk,
                             void* dwq, void* dwk, void* workspace, size_t workspace_size, int dtype) {
    return qknorm_backward_impl(dq_out, dk_out, q, k, wq, wk, N, D, eps, stream, rstd_q, rstd_k, dq, dk, dwq, dwk,
                                workspace, workspace_size, dtype, true);
}

size_t lnmod_qknorm_backward_workspace_bytes(int64_t N, int64_t D) {
    if (N < 0 || N >= (int64_t(1) << 31)) return 0;
    if (D < 8 || D > lnmod::kMaxD || D % 4 != 0) return 0;
    return qknorm_workspace_bytes(N, D);
}

int lnmod_quantize(const void* x, int64_t N, int64_t D, int64_t group, void* stream, void* codes,
                   float* code_scales, int dtype, int code) {
    const int st = check_rows(N, D, group, dtype, code);
    if (st != LNMOD_OK) return st;
    if (N == 0) return LNMOD_OK;
    if (!x || !codes || !code_scales) return LNMOD_EINVAL;
    if (!aligned16(x) || !aligned16(codes)) return LNMOD_EALIGN;
    const hipError_t e = lnmod::launch_quantize(dtype, code, x, N, D, group, codes, code_scales, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? LNMOD_OK : LNMOD_ELAUNCH;
}

int lnmod_dequantize(const void* codes, const float* code_scales, int64_t N, int64_t D, int64_t group, void* stream,
                     void* x, int dtype, int code) {
    const int st = check_rows(N, D, group == 0 ? 32 : group, dtype, code);
    if (st != LNMOD_OK) return st;
    if (N == 0) return LNMOD_OK;
    if (!x || !codes || !code_scales) return LNMOD_EINVAL;
    if (!aligned16(x) || !aligned16(codes)) return LNMOD_EALIGN;
    const hipError_t e = lnmod::launch_dequantize(dtype, code, codes, code_scales, N, D, group, x, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? LNMOD_OK : LNMOD_ELAUNCH;
}

int lnmod_forward_ckpt(const void* x, const void* shift, const void* scale, const int32_t* cu_seqlens,
                       int64_t B_or_nseg, int64_t S_or_T, int64_t D, float eps, int64_t group, void* stream, void* y,
                       void* codes, float* code_scales, float* mean, float* rstd, int dtype, int mod, int code) {
    int64_t S, T;
    if (!gated_shape(cu_seqlens, B_or_nseg, S_or_T, &S, &T)) return LNMOD_EINVAL;
    if (mod != LNMOD_PER_SAMPLE && (mod != LNMOD_PER_TOKEN || cu_seqlens)) return LNMOD_EINVAL;
    if (!valid_group(group) || !valid_code(code)) return LNMOD_EINVAL;
    const int st = check_shape(B_or_nseg, S_or_T, D, eps, dtype, T);
    if (st != LNMOD_OK) return st;
    if (D % 8 != 0) return LNMOD_EUNSUPPORTED;
    if (T == 0) return LNMOD_OK;
    if (B_or_nseg == 0) return LNMOD_EINVAL;
    if (!x || !shift || !scale || !y || !codes || !code_scales || !mean || !rstd) return LNMOD_EINVAL;
    if (!aligned16(x) || !aligned16(shift) || !aligned16(scale) || !aligned16(y) || !aligned16(codes)) return LNMOD_EALIGN;
    const Problem p{dtype, cu_seqlens, B_or_nseg, S, T, D, eps};
    const hipError_t e = lnmod::launch_ckpt_fwd(p, mod == LNMOD_PER_TOKEN, x, shift, scale, y, {codes, code_scales, group},
                                                code, mean, rstd, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? LNMOD_OK : LNMOD_ELAUNCH;
}

int lnmod_backward_ckpt(const void* dy, const void* codes, const float* code_scales, const void* scale,
                        const int32_t* cu_seqlens, int64_t B_or_nseg, int64_t S_or_T, int64_t D, int64_t group,
                        void* stream, const float* mean, const float* rstd, void* dx, void* dshift, void* dscale,
                        void* workspace, size_t workspace_size, int dtype, int mod, int code, int io_grads) {
    int64_t S, T;
    if (!gated_shape(cu_seqlens, B_or_nseg, S_or_T, &S, &T)) return LNMOD_EINVAL;
    if (mod != LNMOD_PER_SAMPLE && (mod != LNMOD_PER_TOKEN || cu_seqlens)) return LNMOD_EINVAL;
    if (!valid_group(group) || !valid_code(code)) return LNMOD_EINVAL;
    const int st = check_shape(B_or_nseg, S_or_T, D, 1.0f, dtype, T);
    if (st != LNMOD_OK) return st;
    if (D % 8 != 0) return LNMOD_EUNSUPPORTED;
    const bool token = mod == LNMOD_PER_TOKEN;
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    if (T == 0) {
        if (token || B_or_nseg == 0) return LNMOD_OK;
        if (!dshift || !dscale) return LNMOD_EINVAL;               // empty sums are zeros
        if (!aligned16(dshift) || !aligned16(dscale)) return LNMOD_EALIGN;
        const int64_t n = grad_floats(B_or_nseg * D, dtype, io_grads != 0);
        hipError_t e = lnmod::launch_zero_f32(static_cast<float*>(dshift), n, hs);
        if (e == hipSuccess) e = lnmod::launch_zero_f32(static_cast<float*>(dscale), n, hs);
        return e == hipSuccess ? LNMOD_OK : LNMOD_ELAUNCH;
    }
    if (B_or_nseg == 0) return LNMOD_EINVAL;
    if (!dy || !codes || !code_scales || !scale || !mean || !rstd || !dx || !dshift || !dscale) return LNMOD_EINVAL;
    if (!aligned16(dy) || !aligned16(codes) || !aligned16(scale) || !aligned16(dx) || !aligned16(dshift) || !aligned16(dscale))
        return LNMOD_EALIGN;
    if (!token) {
        if (!workspace || workspace_size < ckpt_workspace_bytes(B_or_nseg, T, D)) return LNMOD_EWORKSPACE;
        if (!aligned16(workspace)) return LNMOD_EALIGN;
    }
    const Problem p{dtype, cu_seqlens, B_or_nseg, S, T, D, 1.0f};
    const hipError_t e = lnmod::launch_ckpt_bwd(p, token, dy, {const_cast<void*>(codes), const_cast<float*>(code_scales), group},
                                                code, scale, mean, rstd, dx, dshift, dscale, io_grads != 0,
                                                static_cast<float*>(workspace), hs);
    return e == hipSuccess ? LNMOD_OK : LNMOD_ELAUNCH;
}

size_t lnmod_backward_ckpt_workspace_bytes(int64_t B_or_nseg, int64_t total, int64_t D) {
    if (B_or_nseg < 0 || total < 0 || total >= (int64_t(1) << 31)) return 0;
    if (D < 8 || D > lnmod::kMaxD || D % 8 != 0) return 0;
    return ckpt_workspace_bytes(B_or_nseg, total, D);
}

int lnmod_rmsnorm_quant_forward(const void* x, const void* r, const void* w, int64_t N, int64_t D, float eps,
                                int64_t group, void* stream, void* h, void* codes, float* code_scales, void* y,
                                float* rstd, int dtype, int code) {
    if ((group != 0 && !valid_group(group)) || !valid_code(code)) return LNMOD_EINVAL;
    const int st = check_shape(1, N, D, eps, dtype, N);
    if (st != LNMOD_OK) return st;
    if (D % 8 != 0 || (group == 0 && eps < 1e-20f)) return LNMOD_EUNSUPPORTED;
    if (N == 0) return LNMOD_OK;
    if (!x || !w || !rstd || (r == nullptr) != (h == nullptr)) return LNMOD_EINVAL;
    if ((codes == nullptr) == (y == nullptr) || (codes == nullptr) != (code_scales == nullptr)) return LNMOD_EINVAL;
    if (!aligned16(x) || !aligned16(r) || !aligned16(w) || !aligned16(h) || !aligned16(codes) || !aligned16(y))
        return LNMOD_EALIGN;
    const hipError_t e = lnmod::launch_rmsq_fwd(dtype, code, x, r, w, N, D, eps, group, h, y ? y : codes, code_scales, rstd,
                                                y != nullptr, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? LNMOD_OK : LNMOD_ELAUNCH;
}

int lnmod_rmsnorm_quant_backward(const void* dy, const void* dh, const void* h, const void* w, int64_t N, int64_t D,
                                 void* stream, const float* rstd, void* dx, void* dw, void* workspace,
                                 size_t workspace_size, int dtype, int io_grads) {
    return rmsnorm_quant_backward_impl(dy, dh, h, w, N, D, stream, rstd, dx, nullptr, dw, workspace, workspace_size, dtype,
                                       io_grads);
}

int lnmod_rmsnorm_quant_backward_residual(const void* dy, const void* dh, const void* h, const void* w, int64_t N, int64_t D,
                                          void* stream, const float* rstd, void* dx, void* dr, void* dw, void* workspace,
                                          size_t workspace_size, int dtype, int io_grads) {
    if (N > 0 && !dr) return LNMOD_EINVAL;
    return rmsnorm_quant_backward_impl(dy, dh, h, w, N, D, stream, rstd, dx, dr, dw, workspace, workspace_size, dtype, io_grads);
}

size_t lnmod_rmsnorm_quant_backward_workspace_bytes(int64_t N, int64_t D) {
    if (N < 0 || N >= (int64_t(1) << 31)) return 0;
    if (D < 8 || D > lnmod::kMaxD || D % 8 != 0) return 0;
    return rmsq_workspace_bytes(N, D);
}

}  // extern "C"
