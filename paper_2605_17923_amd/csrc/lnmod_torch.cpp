// lnmod_torch.cpp -- the host path of the autograd functions and of the plain forward in C++: checks,
// output and workspace allocation, the call through the C ABI and the autograd node.
//
// Why: a step (forward, autograd, backward) took 80 to 200 us of host time per call in Python -- the
// autograd engine handing the interpreter lock to its own thread, torch.empty nine times, ctypes with
// up to twenty arguments, per-tensor checks -- where its kernels take 18 us on 512 x 1536 fp32 rows and
// 100 us on 32 760 x 1536 bf16 rows, so everything up to about 200 MB per step waited for the host.
//
// Nothing is decided here that the Python binding does not decide: whatever is not the plain case (any
// check that fails, a tensor subclass, functorch, a dispatch mode, a tracer, another current device, a
// status other than LNMOD_OK) goes back to the Python path, which raises its own errors.  The kernels,
// their arguments and the saved tensors with their order are the same either way.
#include <torch/extension.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_cpp_function.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>
#include <ATen/hip/EmptyTensor.h>
#include <ATen/hip/impl/HIPStreamMasqueradingAsCUDA.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <torch/version.h>

#include "lnmod.h"

namespace {

using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

struct NotPlain {};      // thrown to leave a call to the Python path; nothing has been launched

// ---- what counts as the plain case ---------------------------------------------------------------
const c10::DispatchKeySet kSpecial({c10::DispatchKey::Python, c10::DispatchKey::FuncTorchBatched,
                                    c10::DispatchKey::FuncTorchGradWrapper, c10::DispatchKey::Functionalize,
                                    c10::DispatchKey::ZeroTensor, c10::DispatchKey::Negative,
                                    c10::DispatchKey::Conjugate});

bool plain_state() {
    if (c10::impl::TorchDispatchModeTLS::any_modes_set()) return false;
    if (torch::jit::tracer::isTracing()) return false;
    return !c10::impl::tls_local_dispatch_key_set().included_.has(c10::DispatchKey::FuncTorchDynamicLayerFrontMode);
}

// A tensor of exactly torch's own type (or a Parameter), without a forward-mode tangent.
bool plain_object(const py::object& o) {
    return THPVariable_CheckExact(o.ptr()) && !THPVariable_Unpack(o.ptr())._fw_grad(0).defined();
}

bool plain(const Tensor& t, at::IntArrayRef shape, at::ScalarType type, const at::Device& dev) {
    return t.defined() && t.layout() == at::kStrided && t.device() == dev && t.scalar_type() == type &&
           !(t.key_set() & kSpecial).has_any(kSpecial) && t.sizes() == shape && t.is_contiguous();
}

// x itself: on the current device, an element type the kernels know
bool plain_first(const Tensor& x) {
    return x.defined() && x.is_cuda() && (x.scalar_type() == at::kBFloat16 || x.scalar_type() == at::kFloat) &&
           x.device().index() == c10::hip::current_device() && plain(x, x.sizes(), x.scalar_type(), x.device());
}

int code_of(const Tensor& x) { return x.scalar_type() == at::kBFloat16 ? LNMOD_BF16 : LNMOD_F32; }

void* stream_of(const Tensor& x) {
    return c10::hip::getCurrentHIPStreamMasqueradingAsCUDA(x.device().index()).stream();
}

const void* ptr(const Tensor& t) { return t.defined() ? t.const_data_ptr() : nullptr; }
void* out(const Tensor& t) { return t.mutable_data_ptr(); }
const int32_t* cu_ptr(const Tensor& cu) { return cu.defined() ? cu.const_data_ptr<int32_t>() : nullptr; }
const float* f32(const Tensor& t) { return t.defined() ? t.const_data_ptr<float>() : nullptr; }
float* f32_out(const Tensor& t) { return t.mutable_data_ptr<float>(); }

// The batch of a call: [B, S, D], or [T, D] with cu_seqlens.
struct Batch {
    int64_t n, s_or_t, T, D;
    bool ok;
};

Batch batch_of(const Tensor& x, const Tensor& cu) {
    if (!cu.defined()) {
        if (x.dim() != 3) return {0, 0, 0, 0, false};
        return {x.size(0), x.size(1), x.size(0) * x.size(1), x.size(2), true};
    }
    if (x.dim() != 2 || cu.dim() != 1 || cu.numel() < 1 || !plain(cu, cu.sizes(), at::kInt, x.device()))
        return {0, 0, 0, 0, false};
    return {cu.numel() - 1, x.size(0), x.size(0), x.size(1), true};
}

at::TensorOptions f32_like(const Tensor& x) { return x.options().dtype(at::kFloat); }

Tensor scratch(size_t bytes, const Tensor& x) {
    return at::empty({static_cast<int64_t>(bytes < 16 ? 16 : bytes)}, x.options().dtype(at::kByte));
}

// ---- the Python path, for a backward that is not the plain case ------------------------------------
py::object to_python(const Tensor& t) { return t.defined() ? py::cast(t) : py::none(); }
py::object to_python(double v) { return py::float_(v); }
py::object to_python(int64_t v) { return py::int_(v); }
py::object to_python(const std::vector<int64_t>& v) { return py::cast(v); }

// name(args...) of functional.py, with None for an undefined tensor.  Runs on a thread of the autograd engine,
// without the interpreter lock: no Python object is made before it is taken here.  The function's exception (a ValueError of a check, an LnmodError) is kept
// alive across the engine's threads
template <typename... A>
variable_list python_backward(const char* name, size_t outputs, const A&... args) {
    py::gil_scoped_acquire gil;
    try {
        py::tuple r = py::module_::import("paper_2605_17923_amd.functional").attr(name)(to_python(args)...);
        variable_list got;
        for (size_t i = 0; i < outputs; ++i) got.push_back(r[i].cast<Tensor>());
        return got;
    } catch (py::error_already_set& e) {
        e.restore();
        python_error err;
        err.persist();
        throw err;
    }
}

// ---- LayerNorm-Modulate ------------------------------------------------------------------------------
bool ln_shapes(const Tensor& x, const Tensor& scale, const Tensor& cu, Batch* b, bool* token) {
    if (!plain_first(x)) return false;
    *b = batch_of(x, cu);
    if (!b->ok || !scale.defined()) return false;
    *token = !cu.defined() && scale.dim() == 3;
    const int64_t rows[] = {b->n, b->D};
    return plain(scale, *token ? x.sizes() : at::IntArrayRef(rows, 2), x.scalar_type(), x.device());
}

// y and the statistics; throws NotPlain
std::tuple<Tensor, Tensor, Tensor> ln_forward(const Tensor& x, const Tensor& shift, const Tensor& scale,
                                              const Tensor& cu, double eps) {
    Batch b;
    bool token;
    if (!ln_shapes(x, scale, cu, &b, &token) || !plain(shift, scale.sizes(), x.scalar_type(), x.device()))
        throw NotPlain();
    Tensor y = at::empty_like(x);
    Tensor mean = cu.defined() ? at::empty({b.T}, f32_like(x)) : at::empty({b.n, b.s_or_t}, f32_like(x));
    Tensor rstd = at::empty_like(mean);
    const float e = static_cast<float>(eps);
    const int st = cu.defined() ? lnmod_forward_varlen(ptr(x), ptr(shift), ptr(scale), cu_ptr(cu), b.n, b.T, b.D, e,
                                                       stream_of(x), out(y), f32_out(mean), f32_out(rstd), code_of(x))
                                : lnmod_forward(ptr(x), ptr(shift), ptr(scale), b.n, b.s_or_t, b.D, e, stream_of(x),
                                                out(y), f32_out(mean), f32_out(rstd), code_of(x),
                                                token ? LNMOD_PER_TOKEN : LNMOD_PER_SAMPLE);
    if (st != LNMOD_OK) throw NotPlain();
    return {y, mean, rstd};
}

struct LnModulate : public torch::autograd::Function<LnModulate> {
    static Tensor forward(AutogradContext* ctx, const Tensor& x, const Tensor& shift, const Tensor& scale,
                          const std::optional<Tensor>& cu_seqlens, double eps, bool save_stats) {
        const Tensor cu = cu_seqlens.value_or(Tensor());
        auto [y, mean, rstd] = ln_forward(x, shift, scale, cu, eps);
        ctx->saved_data["eps"] = eps;
        if (!save_stats) mean = rstd = Tensor();          // the backward forms them again from x
        ctx->save_for_backward({x, scale, cu, mean, rstd});
        return y;
    }

    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        const variable_list s = ctx->get_saved_variables();
        const Tensor &x = s[0], &scale = s[1], &cu = s[2], &mean = s[3], &rstd = s[4];
        const double eps = ctx->saved_data["eps"].toDouble();
        const Tensor dy = grads[0].contiguous();
        Batch b;
        bool token = false;
        if (plain_state() && ln_shapes(x, scale, cu, &b, &token) && plain(dy, x.sizes(), x.scalar_type(), x.device()) &&
            mean.defined() == rstd.defined() &&
            (!mean.defined() || (plain(mean, mean.sizes(), at::kFloat, x.device()) && mean.numel() == b.T &&
                                 plain(rstd, mean.sizes(), at::kFloat, x.device())))) {
            // With a modulation row per token dshift equals dy, but it is a tensor of its own: a leaf's .grad, a hook or
            // torch.autograd.grad's caller may write to it, and whether dy's memory has another user cannot be told here
            // (a view in front of the operator gives dy a fresh tensor over memory that is still the caller's).
            Tensor dx = at::empty_like(x), dshift = at::empty_like(scale), dscale = at::empty_like(scale);
            int st;
            if (token) {
                st = lnmod_backward(ptr(dy), ptr(x), nullptr, ptr(scale), b.n, b.s_or_t, b.D, static_cast<float>(eps),
                                    stream_of(x), f32(mean), f32(rstd), out(dx), out(dshift), out(dscale), nullptr, 0,
                                    code_of(x), LNMOD_PER_TOKEN);
            } else {
                const Tensor ws = scratch(lnmod_backward_workspace_bytes(b.n, b.T, b.D, LNMOD_PER_SAMPLE), x);
                st = lnmod_backward_io(ptr(dy), ptr(x), ptr(scale), cu_ptr(cu), b.n, b.s_or_t, b.D,
                                       static_cast<float>(eps), stream_of(x), f32(mean), f32(rstd), out(dx),
                                       out(dshift), out(dscale), out(ws), static_cast<size_t>(ws.numel()), code_of(x));
            }
            if (st == LNMOD_OK) return {dx, dshift, dscale, Tensor(), Tensor(), Tensor()};
        }
        variable_list r = python_backward("_ln_backward", 3, dy, x, scale, cu, mean, rstd, eps);
        return {r[0], r[1], r[2], Tensor(), Tensor(), Tensor()};
    }
};

// ---- gated residual + LayerNorm-Modulate ---------------------------------------------------------------
bool gated_shapes(const Tensor& x, const Tensor& u, const Tensor& gate, const Tensor& scale, const Tensor& cu, Batch* b) {
    if (!plain_first(x)) return false;
    *b = batch_of(x, cu);
    const int64_t rows[] = {b->n, b->D};
    const auto mod = at::IntArrayRef(rows, 2);
    return b->ok && plain(u, x.sizes(), x.scalar_type(), x.device()) && plain(gate, mod, x.scalar_type(), x.device()) &&
           plain(scale, mod, x.scalar_type(), x.device());
}

struct GatedLnModulate : public torch::autograd::Function<GatedLnModulate> {
    static variable_list forward(AutogradContext* ctx, const Tensor& x, const Tensor& u, const Tensor& gate,
                                 const Tensor& shift, const Tensor& scale, const std::optional<Tensor>& cu_seqlens,
                                 double eps) {
        const Tensor cu = cu_seqlens.value_or(Tensor());
        Batch b;
        if (!gated_shapes(x, u, gate, scale, cu, &b) || !plain(shift, scale.sizes(), x.scalar_type(), x.device()))
            throw NotPlain();
        Tensor h = at::empty_like(x), y = at::empty_like(x);
        Tensor mean = at::empty({b.T}, f32_like(x)), rstd = at::empty({b.T}, f32_like(x));
        const int st = lnmod_gated_forward(ptr(x), ptr(u), ptr(gate), ptr(shift), ptr(scale), cu_ptr(cu), b.n, b.s_or_t,
                                           b.D, static_cast<float>(eps), stream_of(x), out(h), out(y), f32_out(mean),
                                           f32_out(rstd), code_of(x));
        if (st != LNMOD_OK) throw NotPlain();
        ctx->saved_data["eps"] = eps;
        ctx->save_for_backward({h, u, gate, scale, cu, mean, rstd});
        return {h, y};
    }

    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        const variable_list s = ctx->get_saved_variables();
        const Tensor &h = s[0], &u = s[1], &gate = s[2], &scale = s[3], &cu = s[4], &mean = s[5], &rstd = s[6];
        const double eps = ctx->saved_data["eps"].toDouble();
        const Tensor dh = grads[0].contiguous(), dy = grads[1].contiguous();
        Batch b;
        if (plain_state() && gated_shapes(h, u, gate, scale, cu, &b) &&
            plain(dh, h.sizes(), h.scalar_type(), h.device()) && plain(dy, h.sizes(), h.scalar_type(), h.device()) &&
            plain(mean, at::IntArrayRef(&b.T, 1), at::kFloat, h.device()) &&
            plain(rstd, at::IntArrayRef(&b.T, 1), at::kFloat, h.device())) {
            Tensor dx = at::empty_like(h), du = at::empty_like(h);
            Tensor dgate = at::empty_like(gate), dshift = at::empty_like(gate), dscale = at::empty_like(gate);
            const Tensor ws = scratch(lnmod_gated_backward_workspace_bytes(b.n, b.T, b.D), h);
            const int st = lnmod_gated_backward_io(
                ptr(dy), ptr(dh), ptr(h), ptr(u), ptr(gate), ptr(scale), cu_ptr(cu), b.n, b.s_or_t, b.D,
                static_cast<float>(eps), stream_of(h), f32(mean), f32(rstd), out(dx), out(du), out(dgate), out(dshift),
                out(dscale), out(ws), static_cast<size_t>(ws.numel()), code_of(h));
            if (st == LNMOD_OK) return {dx, du, dgate, dshift, dscale, Tensor(), Tensor()};
        }
        variable_list r = python_backward("_gated_backward", 5, dy, dh, h, u, gate, scale, mean, rstd, cu, eps);
        r.resize(7);
        return r;
    }
};

// ---- Q-Norm + K-Norm -------------------------------------------------------------------------------------
bool qk_shapes(const Tensor& q, const Tensor& k, const Tensor& wq, const Tensor& wk, int64_t* N, int64_t* D) {
    if (!plain_first(q) || q.dim() < 1) return false;
    *D = q.size(-1);
    *N = q.numel() / (*D > 0 ? *D : 1);
    const auto w = at::IntArrayRef(D, 1);
    return plain(k, q.sizes(), q.scalar_type(), q.device()) && plain(wq, w, q.scalar_type(), q.device()) &&
           plain(wk, w, q.scalar_type(), q.device());
}

struct QkNorm : public torch::autograd::Function<QkNorm> {
    static variable_list forward(AutogradContext* ctx, const Tensor& q, const Tensor& k, const Tensor& wq,
                                 const Tensor& wk, double eps) {
        int64_t N, D;
        if (!qk_shapes(q, k, wq, wk, &N, &D)) throw NotPlain();
        Tensor qn = at::empty_like(q), kn = at::empty_like(k);
        Tensor rq = at::empty({N}, f32_like(q)), rk = at::empty({N}, f32_like(q));
        const int st = lnmod_qknorm_forward(ptr(q), ptr(k), ptr(wq), ptr(wk), N, D, static_cast<float>(eps),
                                            stream_of(q), out(qn), out(kn), f32_out(rq), f32_out(rk), code_of(q));
        if (st != LNMOD_OK) throw NotPlain();
        ctx->saved_data["eps"] = eps;
        ctx->save_for_backward({q, k, wq, wk, rq, rk});
        return {qn, kn};
    }

    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        const variable_list s = ctx->get_saved_variables();
        const Tensor &q = s[0], &k = s[1], &wq = s[2], &wk = s[3], &rq = s[4], &rk = s[5];
        const double eps = ctx->saved_data["eps"].toDouble();
        const Tensor dqn = grads[0].contiguous(), dkn = grads[1].contiguous();
        int64_t N, D;
        if (plain_state() && qk_shapes(q, k, wq, wk, &N, &D) && plain(dqn, q.sizes(), q.scalar_type(), q.device()) &&
            plain(dkn, q.sizes(), q.scalar_type(), q.device()) &&
            plain(rq, at::IntArrayRef(&N, 1), at::kFloat, q.device()) &&
            plain(rk, at::IntArrayRef(&N, 1), at::kFloat, q.device())) {
            Tensor dq = at::empty_like(q), dk = at::empty_like(k), dwq = at::empty_like(wq), dwk = at::empty_like(wk);
            const Tensor ws = scratch(lnmod_qknorm_backward_workspace_bytes(N, D), q);
            const int st = lnmod_qknorm_backward_io(ptr(dqn), ptr(dkn), ptr(q), ptr(k), ptr(wq), ptr(wk), N, D,
                                                    static_cast<float>(eps), stream_of(q), f32(rq), f32(rk), out(dq),
                                                    out(dk), out(dwq), out(dwk), out(ws),
                                                    static_cast<size_t>(ws.numel()), code_of(q));
            if (st == LNMOD_OK) return {dq, dk, dwq, dwk, Tensor()};
        }
        variable_list r = python_backward("_qk_backward", 4, dqn, dkn, q, k, wq, wk, rq, rk, eps);
        r.resize(5);
        return r;
    }
};

// ---- activations in 8 bits -------------------------------------------------------------------------------------
// at::empty without the dispatcher (one token, four outputs: 7.2 -> 6.4 us on the host)
Tensor fresh(at::IntArrayRef shape, at::ScalarType type, const Tensor& like) {
    return at::detail::empty_cuda(shape, type, like.device(), std::nullopt);
}
Tensor fresh_like(const Tensor& t) { return fresh(t.sizes(), t.scalar_type(), t); }

Tensor fresh_bytes(size_t bytes, const Tensor& like) { return fresh(static_cast<int64_t>(bytes < 16 ? 16 : bytes), at::kByte, like); }

bool is_group(int64_t group) { return group == 32 || group == 64 || group == 128; }

at::ScalarType type_of_code(int code) { return code == LNMOD_INT8 ? at::kChar : at::kFloat8_e4m3fn; }

bool plain_codes(const Tensor& codes, at::IntArrayRef shape, const at::Device& dev) {
    return codes.defined() && (codes.scalar_type() == at::kChar || codes.scalar_type() == at::kFloat8_e4m3fn) &&
           plain(codes, shape, codes.scalar_type(), dev);
}
int code_of_codes(const Tensor& codes) { return codes.scalar_type() == at::kChar ? LNMOD_INT8 : LNMOD_E4M3; }

// one scale per group of the last dimension; group 0: one per row
std::vector<int64_t> scales_shape(at::IntArrayRef shape, int64_t group) {
    std::vector<int64_t> s = shape.vec();
    if (group == 0) s.pop_back();
    else s.back() = (s.back() + group - 1) / group;
    return s;
}

int64_t rows_of(const Tensor& t) {
    const int64_t D = t.size(-1);
    return t.numel() / (D > 0 ? D : 1);
}

variable_list quantize_call(const Tensor& x, int code, int64_t group) {
    if (!plain_first(x) || x.dim() < 1 || !is_group(group)) throw NotPlain();
    Tensor codes = fresh(x.sizes(), type_of_code(code), x);
    Tensor scales = fresh(scales_shape(x.sizes(), group), at::kFloat, x);
    if (lnmod_quantize(ptr(x), rows_of(x), x.size(-1), group, stream_of(x), out(codes), f32_out(scales), code_of(x), code) != LNMOD_OK)
        throw NotPlain();
    return {codes, scales};
}

variable_list dequantize_call(const Tensor& codes, const Tensor& scales, at::ScalarType type, int64_t group) {
    if (!codes.defined() || !codes.is_cuda() || codes.device().index() != c10::hip::current_device() || codes.dim() < 1 ||
        !plain_codes(codes, codes.sizes(), codes.device()) || !(group == 0 || is_group(group)) ||
        !plain(scales, scales_shape(codes.sizes(), group), at::kFloat, codes.device()) || (type != at::kBFloat16 && type != at::kFloat))
        throw NotPlain();
    Tensor x = fresh(codes.sizes(), type, codes);
    if (lnmod_dequantize(ptr(codes), f32(scales), rows_of(codes), codes.size(-1), group, stream_of(codes), out(x), code_of(x),
                         code_of_codes(codes)) != LNMOD_OK)
        throw NotPlain();
    return {x};
}

// y, codes, scales, mean, rstd; throws NotPlain
variable_list ckpt_forward(const Tensor& x, const Tensor& shift, const Tensor& scale, const Tensor& cu, double eps, int code,
                           int64_t group) {
    Batch b;
    bool token;
    if (!is_group(group) || !ln_shapes(x, scale, cu, &b, &token) || !plain(shift, scale.sizes(), x.scalar_type(), x.device()))
        throw NotPlain();
    Tensor y = fresh_like(x), codes = fresh(x.sizes(), type_of_code(code), x);
    Tensor scales = fresh(scales_shape(x.sizes(), group), at::kFloat, x);
    Tensor mean = fresh(x.sizes().slice(0, x.dim() - 1), at::kFloat, x), rstd = fresh_like(mean);
    const int st = lnmod_forward_ckpt(ptr(x), ptr(shift), ptr(scale), cu_ptr(cu), b.n, b.s_or_t, b.D, static_cast<float>(eps),
                                      group, stream_of(x), out(y), out(codes), f32_out(scales), f32_out(mean), f32_out(rstd),
                                      code_of(x), token ? LNMOD_PER_TOKEN : LNMOD_PER_SAMPLE, code);
    if (st != LNMOD_OK) throw NotPlain();
    return {y, codes, scales, mean, rstd};
}

struct LnModulateCkpt : public torch::autograd::Function<LnModulateCkpt> {
    static Tensor forward(AutogradContext* ctx, const Tensor& x, const Tensor& shift, const Tensor& scale,
                          const std::optional<Tensor>& cu_seqlens, double eps, int64_t code, int64_t group) {
        const Tensor cu = cu_seqlens.value_or(Tensor());
        const variable_list r = ckpt_forward(x, shift, scale, cu, eps, static_cast<int>(code), group);
        ctx->saved_data["group"] = group;
        ctx->save_for_backward({r[1], r[2], scale, cu, r[3], r[4]});
        return r[0];
    }

    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        const variable_list s = ctx->get_saved_variables();
        const Tensor &codes = s[0], &scales = s[1], &scale = s[2], &cu = s[3], &mean = s[4], &rstd = s[5];
        const int64_t group = ctx->saved_data["group"].toInt();
        const Tensor dy = grads[0].contiguous();
        Batch b;
        bool token = false;
        if (plain_state() && ln_shapes(dy, scale, cu, &b, &token) && plain_codes(codes, dy.sizes(), dy.device()) &&
            plain(scales, scales_shape(dy.sizes(), group), at::kFloat, dy.device()) &&
            plain(mean, dy.sizes().slice(0, dy.dim() - 1), at::kFloat, dy.device()) &&
            plain(rstd, mean.sizes(), at::kFloat, dy.device())) {
            Tensor dx = fresh_like(dy), dshift = fresh_like(scale), dscale = fresh_like(scale), ws;
            if (!token) ws = fresh_bytes(lnmod_backward_ckpt_workspace_bytes(b.n, b.T, b.D), dy);
            const int st = lnmod_backward_ckpt(ptr(dy), ptr(codes), f32(scales), ptr(scale), cu_ptr(cu), b.n, b.s_or_t, b.D,
                                               group, stream_of(dy), f32(mean), f32(rstd), out(dx), out(dshift), out(dscale),
                                               token ? nullptr : out(ws), token ? 0 : static_cast<size_t>(ws.numel()),
                                               code_of(dy), token ? LNMOD_PER_TOKEN : LNMOD_PER_SAMPLE,
                                               code_of_codes(codes), 1);
            if (st == LNMOD_OK) return {dx, dshift, dscale, Tensor(), Tensor(), Tensor(), Tensor()};
        }
        variable_list r = python_backward("_ckpt_backward", 3, dy, codes, scales, scale, mean, rstd, cu, group);
        r.resize(7);
        return r;
    }
};

bool rms_shapes(const Tensor& x, const Tensor& w, const Tensor& other, int64_t* N, int64_t* D) {
    if (!plain_first(x) || x.dim() < 1) return false;
    *D = x.size(-1);
    *N = rows_of(x);
    return plain(w, at::IntArrayRef(D, 1), x.scalar_type(), x.device()) &&
           (!other.defined() || plain(other, x.sizes(), x.scalar_type(), x.device()));
}

// codes and scales, or y; then h (x itself without a residual) and rstd; throws NotPlain
variable_list rms_forward(const Tensor& x, const Tensor& w, const Tensor& residual, double eps, int code, int64_t group,
                          bool values) {
    int64_t N, D;
    if (!(group == 0 || is_group(group)) || !rms_shapes(x, w, residual, &N, &D)) throw NotPlain();
    Tensor codes, scales, y, h;
    if (values) {
        y = fresh_like(x);
    } else {
        codes = fresh(x.sizes(), type_of_code(code), x);
        scales = fresh(scales_shape(x.sizes(), group), at::kFloat, x);
    }
    if (residual.defined()) h = fresh_like(x);
    Tensor rstd = fresh(N, at::kFloat, x);
    const int st = lnmod_rmsnorm_quant_forward(ptr(x), ptr(residual), ptr(w), N, D, static_cast<float>(eps), group,
                                               stream_of(x), h.defined() ? out(h) : nullptr, values ? nullptr : out(codes),
                                               values ? nullptr : f32_out(scales), values ? out(y) : nullptr, f32_out(rstd),
                                               code_of(x), code);
    if (st != LNMOD_OK) throw NotPlain();
    if (!h.defined()) h = x;
    return values ? variable_list{y, h, rstd} : variable_list{codes, scales, h, rstd};
}

// dx, dw, dr (dx itself unless it has to be a tensor of its own); empty where the call is not the plain case
variable_list rms_backward(const Tensor& dy, const Tensor& h, const Tensor& w, const Tensor& rstd, const Tensor& dh, bool io_grads,
                           bool own_dr) {
    int64_t N, D;
    if (!rms_shapes(h, w, dh, &N, &D) || !plain(dy, h.sizes(), h.scalar_type(), h.device()) ||
        !plain(rstd, at::IntArrayRef(&N, 1), at::kFloat, h.device()))
        return {};
    Tensor dx = fresh_like(h), dw = fresh(D, io_grads ? h.scalar_type() : at::kFloat, h), dr = own_dr ? fresh_like(h) : dx;
    const Tensor ws = fresh_bytes(lnmod_rmsnorm_quant_backward_workspace_bytes(N, D), h);
    const size_t bytes = static_cast<size_t>(ws.numel());
    const int st = own_dr ? lnmod_rmsnorm_quant_backward_residual(ptr(dy), ptr(dh), ptr(h), ptr(w), N, D, stream_of(h), f32(rstd),
                                                                  out(dx), out(dr), out(dw), out(ws), bytes, code_of(h), io_grads)
                          : lnmod_rmsnorm_quant_backward(ptr(dy), ptr(dh), ptr(h), ptr(w), N, D, stream_of(h), f32(rstd), out(dx),
                                                         out(dw), out(ws), bytes, code_of(h), io_grads);
    return st == LNMOD_OK ? variable_list{dx, dw, dr} : variable_list{};
}

struct RmsNormQuant : public torch::autograd::Function<RmsNormQuant> {
    static variable_list forward(AutogradContext* ctx, const Tensor& x, const Tensor& w, const std::optional<Tensor>& residual,
                                 double eps, int64_t code, int64_t group) {
        const Tensor r = residual.value_or(Tensor());
        const variable_list o = rms_forward(x, w, r, eps, static_cast<int>(code), group, true);
        ctx->saved_data["residual"] = r.defined();
        ctx->save_for_backward({o[1], w, o[2]});
        return r.defined() ? variable_list{o[1], o[0]} : variable_list{o[0]};
    }

    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        const variable_list s = ctx->get_saved_variables();
        const Tensor &h = s[0], &w = s[1], &rstd = s[2];
        const bool residual = ctx->saved_data["residual"].toBool();
        const Tensor dy = grads.back().contiguous(), dh = residual ? grads[0].contiguous() : Tensor();
        // x and the residual get gradients in memory of their own: where views lie in front of the operator, two leaves'
        // .grad would share it, and the next backward, adding to one, would add to both.
        const bool both = residual && ctx->needs_input_grad(0) && ctx->needs_input_grad(2);
        variable_list r;
        if (plain_state()) r = rms_backward(dy, h, w, rstd, dh, true, both);
        if (r.empty()) r = python_backward("_rms_quant_backward", 3, dy, h, w, rstd, dh, static_cast<int64_t>(both));
        return {r[0], r[1], residual ? r[2] : Tensor(), Tensor(), Tensor(), Tensor()};
    }
};

// ---- codes with one scale for a row, and their product ---------------------------------------------------------
variable_list quantize_rows_call(const Tensor& x, int code) {
    if (!plain_first(x) || x.dim() < 1) throw NotPlain();
    Tensor codes = fresh(x.sizes(), type_of_code(code), x);
    Tensor scales = fresh(x.sizes().slice(0, x.dim() - 1), at::kFloat, x);
    if (lnmod_quantize_rows(ptr(x), rows_of(x), x.size(-1), stream_of(x), out(codes), f32_out(scales), code_of(x), code) != LNMOD_OK)
        throw NotPlain();
    return {codes, scales};
}

variable_list code_product_call(const Tensor& codes, const Tensor& scales, const Tensor& w, const Tensor& w_scales,
                                const Tensor& bias, at::ScalarType type) {
    if (!codes.defined() || !codes.is_cuda() || codes.device().index() != c10::hip::current_device() || codes.dim() < 1 ||
        !plain_codes(codes, codes.sizes(), codes.device()) || !w.defined() || w.dim() != 2 || (type != at::kBFloat16 && type != at::kFloat))
        throw NotPlain();
    const at::Device dev = codes.device();
    const int64_t K = codes.size(-1), N = w.size(0);
    const int64_t weight[] = {N, K};
    if (!plain(scales, codes.sizes().slice(0, codes.dim() - 1), at::kFloat, dev) || !plain(w, at::IntArrayRef(weight, 2), codes.scalar_type(), dev) ||
        !plain(w_scales, at::IntArrayRef(&N, 1), at::kFloat, dev) || (bias.defined() && !plain(bias, at::IntArrayRef(&N, 1), type, dev)))
        throw NotPlain();
    std::vector<int64_t> shape = codes.sizes().vec();
    shape.back() = N;
    Tensor y = fresh(shape, type, codes);
    if (lnmod_code_product(ptr(codes), f32(scales), ptr(w), f32(w_scales), ptr(bias), rows_of(codes), N, K, stream_of(codes),
                           out(y), code_of(y), code_of_codes(codes)) != LNMOD_OK)
        throw NotPlain();
    return {y};
}

// ---- rotary positions ------------------------------------------------------------------------------------------
// A tensor [.., tokens, heads, features] as the kernels can read it, or false.
bool heads_of(const Tensor& t, at::IntArrayRef shape, at::ScalarType type, const at::Device& dev, lnmod_heads* h) {
    if (!t.defined() || t.layout() != at::kStrided || t.device() != dev || t.scalar_type() != type ||
        (t.key_set() & kSpecial).has_any(kSpecial) || t.sizes() != shape)
        return false;
    if (t.numel() == 0) {
        *h = {nullptr, 0, 0, 0};
        return true;
    }
    const int64_t step = 16 / static_cast<int64_t>(t.element_size()), n = t.dim();
    if (t.size(-1) > 1 && t.stride(-1) != 1) return false;
    int64_t stride[3] = {0, 0, 0};
    for (int64_t d = 0; d < n - 1; ++d) {
        const int64_t s = t.size(d) == 1 ? 0 : t.stride(d);
        if (s % step != 0) return false;
        stride[d + 4 - n] = s;
    }
    h->data = t.const_data_ptr();
    if (reinterpret_cast<uintptr_t>(h->data) % 16 != 0) return false;
    h->batch = stride[0];
    h->token = stride[1];
    h->head = stride[2];
    return true;
}

// What both operators share.
struct RotaryCall {
    lnmod_heads q, k;
    lnmod_rotation rot;
    int64_t B, S, heads, kv, hd;
};

bool rotary_of(const Tensor& q, const Tensor& k, const Tensor& positions, const Tensor& table, const std::vector<int64_t>& axes,
               bool interleaved, RotaryCall* c) {
    if (!q.defined() || !q.is_cuda() || (q.scalar_type() != at::kBFloat16 && q.scalar_type() != at::kFloat) ||
        q.device().index() != c10::hip::current_device() || (q.dim() != 3 && q.dim() != 4) || axes.empty() || axes.size() > LNMOD_MAX_AXES)
        return false;
    const at::Device dev = q.device();
    std::vector<int64_t> shape = q.sizes().vec();
    c->hd = shape.back();
    c->heads = shape[shape.size() - 2];
    c->kv = 0;
    if (!heads_of(q, shape, q.scalar_type(), dev, &c->q)) return false;
    if (k.defined()) {
        if (k.dim() != q.dim()) return false;
        c->kv = shape[shape.size() - 2] = k.size(-2);
        if (c->kv == 0 || !heads_of(k, shape, q.scalar_type(), dev, &c->k)) return false;
    }
    c->B = q.dim() == 4 ? q.size(0) : 1;
    c->S = q.size(-3);
    if (!positions.defined() || positions.dim() < 2) return false;
    const bool shared = q.dim() == 4 && positions.dim() == 2;
    std::vector<int64_t> rows = q.sizes().slice(shared ? 1 : 0, shared ? 1 : q.dim() - 2).vec();
    rows.push_back(static_cast<int64_t>(axes.size()));
    int64_t width = 0;
    for (const int64_t d : axes) {
        if (d < 2 || d > c->hd) return false;
        width += d;
    }
    if (!plain(positions, rows, at::kInt, dev) || !table.defined() || table.dim() != 3) return false;
    const int64_t entries[] = {table.size(0), width / 2, 2};
    if (!plain(table, at::IntArrayRef(entries, 3), at::kFloat, dev)) return false;
    c->rot = {positions.const_data_ptr<int32_t>(), shared ? c->S : c->B * c->S, f32(table), table.size(0),
              static_cast<int32_t>(axes.size()), {0, 0, 0, 0}, interleaved ? 1 : 0};
    for (size_t i = 0; i < axes.size(); ++i) c->rot.features[i] = static_cast<int32_t>(axes[i]);
    return true;
}

// A gradient as the kernels can read it.
Tensor readable(const Tensor& t) {
    lnmod_heads h;
    return t.defined() && t.layout() == at::kStrided && heads_of(t, t.sizes(), t.scalar_type(), t.device(), &h) ? t : t.contiguous();
}

// both results (the second undefined without k); empty where the call is not the plain case
variable_list rotary_run(const Tensor& q, const Tensor& k, const Tensor& positions, const Tensor& table,
                         const std::vector<int64_t>& axes, bool interleaved, bool inverse) {
    RotaryCall c;
    if (!rotary_of(q, k, positions, table, axes, interleaved, &c)) return {};
    Tensor qo = fresh_like(q), ko = k.defined() ? fresh_like(k) : Tensor();
    const int st = lnmod_rotary(&c.q, k.defined() ? &c.k : nullptr, c.B, c.S, c.heads, c.kv, c.hd, &c.rot, inverse ? 1 : 0,
                                stream_of(q), out(qo), k.defined() ? out(ko) : nullptr, code_of(q));
    return st == LNMOD_OK ? variable_list{qo, ko} : variable_list{};
}

c10::List<int64_t> axes_list(const std::vector<int64_t>& axes) { return c10::List<int64_t>(at::IntArrayRef(axes)); }

struct Rotary : public torch::autograd::Function<Rotary> {
    static variable_list forward(AutogradContext* ctx, const Tensor& q, const std::optional<Tensor>& k, const Tensor& positions,
                                 const Tensor& table, const std::vector<int64_t>& axes, bool interleaved) {
        variable_list r = rotary_run(q, k.value_or(Tensor()), positions, table, axes, interleaved, false);
        if (r.empty()) throw NotPlain();
        ctx->saved_data["axes"] = axes_list(axes);
        ctx->saved_data["interleaved"] = interleaved;
        ctx->save_for_backward({positions, table});
        if (!r[1].defined()) r.pop_back();
        return r;
    }

    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        const variable_list s = ctx->get_saved_variables();
        const std::vector<int64_t> axes = ctx->saved_data["axes"].toIntVector();
        const bool interleaved = ctx->saved_data["interleaved"].toBool();
        const Tensor dq = readable(grads[0]), dk = grads.size() > 1 ? readable(grads[1]) : Tensor();
        variable_list r;
        if (plain_state()) r = rotary_run(dq, dk, s[0], s[1], axes, interleaved, true);
        if (r.empty()) {
            r = python_backward("_rotary_backward", dk.defined() ? 2 : 1, dq, dk, s[0], s[1], axes, static_cast<int64_t>(interleaved));
            r.resize(2);
        }
        return {r[0], r[1], Tensor(), Tensor(), Tensor(), Tensor()};
    }
};

// whether each head has the norm, or its tokens; false where the weights are neither's
bool qk_weights(const Tensor& q, const Tensor& wq, const Tensor& wk, const RotaryCall& c, bool* per_head) {
    if (!wq.defined() || !wk.defined() || wq.dim() != 1 || wk.dim() != 1) return false;
    *per_head = wq.size(0) == c.hd && wk.size(0) == c.hd;
    const int64_t nq = *per_head ? c.hd : c.heads * c.hd, nk = *per_head ? c.hd : c.kv * c.hd;
    return plain(wq, at::IntArrayRef(&nq, 1), q.scalar_type(), q.device()) && plain(wk, at::IntArrayRef(&nk, 1), q.scalar_type(), q.device());
}

// q and k, normed and turned, and 1 / root of both; throws NotPlain
variable_list qk_rotary_forward(const Tensor& q, const Tensor& k, const Tensor& wq, const Tensor& wk, const Tensor& positions,
                                const Tensor& table, const std::vector<int64_t>& axes, bool interleaved, double eps) {
    RotaryCall c;
    bool per_head;
    if (!k.defined() || !rotary_of(q, k, positions, table, axes, interleaved, &c) || !qk_weights(q, wq, wk, c, &per_head)) throw NotPlain();
    const int64_t lead = q.dim() - (per_head ? 1 : 2);
    Tensor qo = fresh_like(q), ko = fresh_like(k);
    Tensor rq = fresh(q.sizes().slice(0, lead), at::kFloat, q), rk = fresh(k.sizes().slice(0, lead), at::kFloat, q);
    const int st = lnmod_qknorm_rotary_forward(&c.q, &c.k, ptr(wq), ptr(wk), c.B, c.S, c.heads, c.kv, c.hd, &c.rot,
                                               static_cast<float>(eps), per_head, stream_of(q), out(qo), out(ko), f32_out(rq),
                                               f32_out(rk), code_of(q));
    if (st != LNMOD_OK) throw NotPlain();
    return {qo, ko, rq, rk};
}

struct QkNormRotary : public torch::autograd::Function<QkNormRotary> {
    static variable_list forward(AutogradContext* ctx, const Tensor& q, const Tensor& k, const Tensor& wq, const Tensor& wk,
                                 const Tensor& positions, const Tensor& table, const std::vector<int64_t>& axes, bool interleaved,
                                 double eps) {
        const variable_list r = qk_rotary_forward(q, k, wq, wk, positions, table, axes, interleaved, eps);
        ctx->saved_data["axes"] = axes_list(axes);
        ctx->saved_data["interleaved"] = interleaved;
        ctx->save_for_backward({q, k, wq, wk, r[2], r[3], positions, table});
        return {r[0], r[1]};
    }

    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        const variable_list s = ctx->get_saved_variables();
        const Tensor &q = s[0], &k = s[1], &wq = s[2], &wk = s[3], &rq = s[4], &rk = s[5], &positions = s[6], &table = s[7];
        const std::vector<int64_t> axes = ctx->saved_data["axes"].toIntVector();
        const bool interleaved = ctx->saved_data["interleaved"].toBool();
        const Tensor dqr = readable(grads[0]), dkr = readable(grads[1]);
        RotaryCall c;
        lnmod_heads gq, gk;
        bool per_head;
        if (plain_state() && rotary_of(q, k, positions, table, axes, interleaved, &c) && qk_weights(q, wq, wk, c, &per_head) &&
            heads_of(dqr, q.sizes(), q.scalar_type(), q.device(), &gq) && heads_of(dkr, k.sizes(), q.scalar_type(), q.device(), &gk) &&
            plain(rq, q.sizes().slice(0, q.dim() - (per_head ? 1 : 2)), at::kFloat, q.device()) &&
            plain(rk, k.sizes().slice(0, k.dim() - (per_head ? 1 : 2)), at::kFloat, q.device())) {
            Tensor dq = fresh_like(q), dk = fresh_like(k), dwq = fresh_like(wq), dwk = fresh_like(wk);
            const Tensor ws = fresh_bytes(lnmod_qknorm_rotary_backward_workspace_bytes(c.B * c.S, c.heads, c.kv, c.hd, per_head), q);
            const int st = lnmod_qknorm_rotary_backward(&gq, &gk, &c.q, &c.k, ptr(wq), ptr(wk), c.B, c.S, c.heads, c.kv, c.hd, &c.rot,
                                                        per_head, stream_of(q), f32(rq), f32(rk), out(dq), out(dk), out(dwq),
                                                        out(dwk), out(ws), static_cast<size_t>(ws.numel()), code_of(q), 1);
            if (st == LNMOD_OK) return {dq, dk, dwq, dwk, Tensor(), Tensor(), Tensor(), Tensor(), Tensor()};
        }
        variable_list r = python_backward("_qk_rotary_backward", 4, dqr, dkr, q, k, wq, wk, rq, rk, positions, table, axes,
                                          static_cast<int64_t>(interleaved));
        r.resize(9);
        return r;
    }
};

// ---- Python entry points: None where the call is left to the Python path ------------------------------------
template <typename F>
py::object attempt(const std::vector<py::object>& tensors, const py::object& cu, F&& call) {
    if (!plain_state()) return py::none();
    for (const auto& o : tensors)
        if (!plain_object(o)) return py::none();
    if (!cu.is_none() && !plain_object(cu)) return py::none();
    variable_list r;
    try {
        // the launch may wait for room in the queue, and saved-tensor hooks take the lock themselves
        py::gil_scoped_release nogil;
        r = call();
    } catch (const NotPlain&) {
        return py::none();
    }
    if (r.size() == 1) return py::cast(r[0]);
    py::tuple t(r.size());
    for (size_t i = 0; i < r.size(); ++i) t[i] = to_python(r[i]);
    return t;
}

const Tensor& unpack(const py::object& o) { return THPVariable_Unpack(o.ptr()); }
std::optional<Tensor> unpack_or(const py::object& o) {
    return o.is_none() ? std::nullopt : std::optional<Tensor>(unpack(o));
}

py::object forward(const py::object& x, const py::object& shift, const py::object& scale, const py::object& cu, double eps) {
    return attempt({x, shift, scale}, cu, [&] {
        auto [y, mean, rstd] = ln_forward(unpack(x), unpack(shift), unpack(scale), unpack_or(cu).value_or(Tensor()), eps);
        return variable_list{y, mean, rstd};
    });
}

py::object ln_modulate(const py::object& x, const py::object& shift, const py::object& scale, const py::object& cu,
                       double eps, bool save_stats) {
    return attempt({x, shift, scale}, cu, [&] {
        return variable_list{LnModulate::apply(unpack(x), unpack(shift), unpack(scale), unpack_or(cu), eps, save_stats)};
    });
}

py::object gated_ln_modulate(const py::object& x, const py::object& u, const py::object& gate, const py::object& shift,
                             const py::object& scale, const py::object& cu, double eps) {
    return attempt({x, u, gate, shift, scale}, cu, [&] {
        return GatedLnModulate::apply(unpack(x), unpack(u), unpack(gate), unpack(shift), unpack(scale), unpack_or(cu), eps);
    });
}

py::object qk_norm(const py::object& q, const py::object& k, const py::object& wq, const py::object& wk, double eps) {
    return attempt({q, k, wq, wk}, py::none(), [&] {
        return QkNorm::apply(unpack(q), unpack(k), unpack(wq), unpack(wk), eps);
    });
}

// the number of "int8" or "e4m3", or -1; the group, or -1
int code_number(const py::object& code) {
    if (!py::isinstance<py::str>(code)) return -1;
    const std::string name = code.cast<std::string>();
    return name == "int8" ? LNMOD_INT8 : name == "e4m3" ? LNMOD_E4M3 : -1;
}
int64_t group_number(const py::object& group) {
    if (!PyLong_CheckExact(group.ptr())) return -1;
    const long v = PyLong_AsLong(group.ptr());
    if (v == -1 && PyErr_Occurred()) PyErr_Clear();
    return v == 0 || is_group(v) ? v : -1;
}

// whether a tensor of a call that is differentiated elsewhere asks for a gradient is no matter here: these calls have none
py::object quantize(const py::object& x, const py::object& code, const py::object& group) {
    const int c = code_number(code);
    const int64_t g = group_number(group);
    if (c < 0 || g < 0) return py::none();
    return attempt({x}, py::none(), [&] { return quantize_call(unpack(x), c, g); });
}

py::object dequantize(const py::object& codes, const py::object& scales, const py::object& dtype, const py::object& group) {
    const int64_t g = group_number(group);
    if (g < 0 || !THPDtype_Check(dtype.ptr())) return py::none();
    const at::ScalarType type = reinterpret_cast<THPDtype*>(dtype.ptr())->scalar_type;
    return attempt({codes, scales}, py::none(), [&] { return dequantize_call(unpack(codes), unpack(scales), type, g); });
}

py::object forward_ckpt(const py::object& x, const py::object& shift, const py::object& scale, const py::object& cu, double eps,
                        const py::object& code, const py::object& group) {
    const int c = code_number(code);
    const int64_t g = group_number(group);
    if (c < 0 || g < 0) return py::none();
    return attempt({x, shift, scale}, cu, [&] {
        return ckpt_forward(unpack(x), unpack(shift), unpack(scale), unpack_or(cu).value_or(Tensor()), eps, c, g);
    });
}

py::object ln_modulate_ckpt(const py::object& x, const py::object& shift, const py::object& scale, const py::object& cu,
                            double eps, const py::object& code, const py::object& group) {
    const int64_t c = code_number(code), g = group_number(group);
    if (c < 0 || g < 0) return py::none();
    return attempt({x, shift, scale}, cu, [&] {
        return variable_list{LnModulateCkpt::apply(unpack(x), unpack(shift), unpack(scale), unpack_or(cu), eps, c, g)};
    });
}

// attempt() checks the optional last tensor as it does cu_seqlens
py::object rmsnorm_quant_forward(const py::object& x, const py::object& w, const py::object& residual, double eps,
                                 const py::object& code, const py::object& group) {
    const int c = code_number(code);
    const int64_t g = group_number(group);
    if (c < 0 || g < 0) return py::none();
    return attempt({x, w}, residual, [&] {
        return rms_forward(unpack(x), unpack(w), unpack_or(residual).value_or(Tensor()), eps, c, g, false);
    });
}

py::object rmsnorm_quant_backward(const py::object& dy, const py::object& h, const py::object& w, const py::object& rstd,
                                  const py::object& dh) {
    return attempt({dy, h, w, rstd}, dh, [&] {
        variable_list r = rms_backward(unpack(dy), unpack(h), unpack(w), unpack(rstd), unpack_or(dh).value_or(Tensor()), false, false);
        if (r.empty()) throw NotPlain();
        r.pop_back();                        // dr is dx
        return r;
    });
}

py::object rms_norm_quant(const py::object& x, const py::object& w, const py::object& residual, double eps,
                          const py::object& code, const py::object& group) {
    const int64_t c = code_number(code), g = group_number(group);
    if (c < 0 || g < 0) return py::none();
    return attempt({x, w}, residual, [&] {
        return RmsNormQuant::apply(unpack(x), unpack(w), unpack_or(residual), eps, c, g);
    });
}

py::object quantize_rows(const py::object& x, const py::object& code) {
    const int c = code_number(code);
    if (c < 0) return py::none();
    return attempt({x}, py::none(), [&] { return quantize_rows_call(unpack(x), c); });
}

// attempt() checks the optional tensor of these calls as it does cu_seqlens
py::object code_product(const py::object& codes, const py::object& scales, const py::object& w, const py::object& w_scales,
                        const py::object& bias, const py::object& dtype) {
    if (!THPDtype_Check(dtype.ptr())) return py::none();
    const at::ScalarType type = reinterpret_cast<THPDtype*>(dtype.ptr())->scalar_type;
    return attempt({codes, scales, w, w_scales}, bias, [&] {
        return code_product_call(unpack(codes), unpack(scales), unpack(w), unpack(w_scales), unpack_or(bias).value_or(Tensor()), type);
    });
}

// the features of each axis; empty where they are no tuple of numbers
std::vector<int64_t> axes_number(const py::object& axes) {
    std::vector<int64_t> v;
    if (!PyTuple_CheckExact(axes.ptr())) return v;
    for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(axes.ptr()); ++i) {
        PyObject* o = PyTuple_GET_ITEM(axes.ptr(), i);
        const long d = PyLong_CheckExact(o) ? PyLong_AsLong(o) : -1;
        if (d == -1 && PyErr_Occurred()) PyErr_Clear();
        if (d < 2) return {};
        v.push_back(d);
    }
    return v;
}

py::object rotary_call(const py::object& q, const py::object& k, const py::object& positions, const py::object& table,
                       const py::object& axes, const py::object& interleaved, bool inverse) {
    const std::vector<int64_t> v = axes_number(axes);
    if (v.empty() || !PyBool_Check(interleaved.ptr())) return py::none();
    return attempt({q, positions, table}, k, [&] {
        variable_list r = rotary_run(unpack(q), unpack_or(k).value_or(Tensor()), unpack(positions), unpack(table), v,
                                     interleaved.ptr() == Py_True, inverse);
        if (r.empty()) throw NotPlain();
        return r;
    });
}

py::object rotary(const py::object& q, const py::object& k, const py::object& positions, const py::object& table,
                  const py::object& axes, const py::object& interleaved) {
    const std::vector<int64_t> v = axes_number(axes);
    if (v.empty() || !PyBool_Check(interleaved.ptr())) return py::none();
    return attempt({q, positions, table}, k, [&] {
        return Rotary::apply(unpack(q), unpack_or(k), unpack(positions), unpack(table), v, interleaved.ptr() == Py_True);
    });
}

py::object qknorm_rotary_forward(const py::object& q, const py::object& k, const py::object& wq, const py::object& wk,
                                 const py::object& positions, const py::object& table, const py::object& axes,
                                 const py::object& interleaved, double eps) {
    const std::vector<int64_t> v = axes_number(axes);
    if (v.empty() || !PyBool_Check(interleaved.ptr())) return py::none();
    return attempt({q, k, wq, wk, positions, table}, py::none(), [&] {
        return qk_rotary_forward(unpack(q), unpack(k), unpack(wq), unpack(wk), unpack(positions), unpack(table), v,
                                 interleaved.ptr() == Py_True, eps);
    });
}

py::object qk_norm_rotary(const py::object& q, const py::object& k, const py::object& wq, const py::object& wk,
                          const py::object& positions, const py::object& table, const py::object& axes,
                          const py::object& interleaved, double eps) {
    const std::vector<int64_t> v = axes_number(axes);
    if (v.empty() || !PyBool_Check(interleaved.ptr())) return py::none();
    return attempt({q, k, wq, wk, positions, table}, py::none(), [&] {
        return QkNormRotary::apply(unpack(q), unpack(k), unpack(wq), unpack(wk), unpack(positions), unpack(table), v,
                                   interleaved.ptr() == Py_True, eps);
    });
}

// ---- what y.grad_fn shows --------------------------------------------------------------------------------------
// The node's Python type, with the saved tensors that the Python classes' nodes show (the same ones in the same order,
// None where nothing was saved; an error once the backward has freed them).
template <typename Op>
PyObject* saved_tensors(PyObject* self, void*) {
    HANDLE_TH_ERRORS
    auto& node = static_cast<torch::autograd::CppNode<Op>&>(*reinterpret_cast<torch::autograd::THPCppFunction*>(self)->cdata);
    const variable_list saved = node.ctx_.get_saved_variables();
    py::tuple t(saved.size());
    for (size_t i = 0; i < saved.size(); ++i) t[i] = to_python(saved[i]);
    return t.release().ptr();
    END_HANDLE_TH_ERRORS
}

template <typename Op>
void register_node(const char* name) {
    using namespace torch::autograd;                   // the property macro names functions of it
    static PyTypeObject type;
    static PyGetSetDef properties[] = {THP_FUNCTION_DEFAULT_PROPERTIES,
                                       {"saved_tensors", saved_tensors<Op>, nullptr, nullptr, nullptr},
                                       {nullptr, nullptr, nullptr, nullptr, nullptr}};
    if (!_initFunctionPyTypeObject(type, name, properties, nullptr)) throw py::error_already_set();
    registerCppFunction(typeid(CppNode<Op>), &type);
}

}  // namespace

PYBIND11_MODULE(TORCH_EXTENSION_NAME, m) {
    m.doc() = "Host path of the lnmod operators; every function returns None for a call it leaves to the Python path.";
    m.attr("built_for") = TORCH_VERSION;
    register_node<LnModulate>("LnModulateBackward");
    register_node<GatedLnModulate>("GatedLnModulateBackward");
    register_node<QkNorm>("QkNormBackward");
    register_node<LnModulateCkpt>("LnModulateCkptBackward");
    register_node<RmsNormQuant>("RmsNormQuantBackward");
    register_node<Rotary>("RotaryBackward");
    register_node<QkNormRotary>("QkNormRotaryBackward");
    m.def("forward", &forward);
    m.def("ln_modulate", &ln_modulate);
    m.def("gated_ln_modulate", &gated_ln_modulate);
    m.def("qk_norm", &qk_norm);
    m.def("quantize", &quantize);
    m.def("dequantize", &dequantize);
    m.def("forward_ckpt", &forward_ckpt);
    m.def("ln_modulate_ckpt", &ln_modulate_ckpt);
    m.def("rmsnorm_quant_forward", &rmsnorm_quant_forward);
    m.def("rmsnorm_quant_backward", &rmsnorm_quant_backward);
    m.def("rms_norm_quant", &rms_norm_quant);
    m.def("quantize_rows", &quantize_rows);
    m.def("code_product", &code_product);
    m.def("rotary_call", &rotary_call);
    m.def("rotary", &rotary);
    m.def("qknorm_rotary_forward", &qknorm_rotary_forward);
    m.def("qk_norm_rotary", &qk_norm_rotary);
}
