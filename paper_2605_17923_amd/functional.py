"""torch.autograd wrappers over the C ABI: the fused operators as differentiable functions.

Everything numerical runs in the HIP kernels; the functions allocate outputs with torch and
keep what the backward needs; the kernels round the float32 sums of the parameter gradients to the
parameters' dtype where they form them.
Inputs must be contiguous CUDA tensors in bfloat16 or float32 (q and k of the rotations may be strided views); work is enqueued on torch's
current stream.  Without the built library every call raises (there is no fallback).

Ordinary calls run the autograd function of the C++ extension module (csrc/lnmod_torch.cpp).  The classes
below are the same functions in Python, for every call that one leaves alone: wrong arguments (they raise
the errors), tensor subclasses, functorch transforms, dispatch modes, tracers.

    y        = ln_modulate(x, shift, scale)                      x [B,S,D]; shift, scale [B,D] or [B,S,D]
    y        = ln_modulate(x, shift, scale, cu_seqlens=cu)       x [T,D] packed; shift, scale [nseg,D]
    h, y     = gated_ln_modulate(x, u, gate, shift, scale)       h = x + gate*u, y = LN(h)(1+scale)+shift
    qn, kn   = qk_norm(q, k, wq, wk)                             RMS norm with weight of q and of k
    y        = ln_modulate_ckpt(x, shift, scale)                 ln_modulate that keeps x in 8 bits for the backward
    y        = rms_norm_quant(x, w)                              RMS norm with weight, rounded to 8 bits and back
    h, y     = rms_norm_quant(x, w, residual)                    h = x + residual first
    qr, kr   = rotary(q, k, positions, table, axes)              rotary positions with several axes
    qr, kr   = qk_norm_rotary(q, k, wq, wk, positions, table, axes)   qk_norm and the rotation in one pass
"""
import torch

from . import lnmod


def _contig(*ts):
    for t in ts:
        if t is not None and not t.is_contiguous():
            raise ValueError("tensors must be contiguous")


def _ln_backward(dy, x, scale, cu_seqlens, mean, rstd, eps):
    if cu_seqlens is not None:
        return lnmod._backward_varlen(dy, x, scale, cu_seqlens, mean, rstd, eps, io_grads=True)
    return lnmod._backward(dy, x, scale, mean, rstd, eps, io_grads=True)


class _LnModulate(torch.autograd.Function):
    """Sec. 3.3: forward saves x, scale and (optionally) the per-token statistics."""

    @staticmethod
    def forward(ctx, x, shift, scale, cu_seqlens, eps, save_stats):
        _contig(x, shift, scale, cu_seqlens)
        if cu_seqlens is None:
            y, mean, rstd = lnmod.forward(x, shift, scale, eps)
        else:
            y, mean, rstd = lnmod.forward_varlen(x, shift, scale, cu_seqlens, eps)
        ctx.eps = eps
        if save_stats:
            ctx.save_for_backward(x, scale, cu_seqlens, mean, rstd)
        else:                                   # the backward forms them again from x
            ctx.save_for_backward(x, scale, cu_seqlens, None, None)
        return y

    @staticmethod
    def backward(ctx, dy):
        x, scale, cu, mean, rstd = ctx.saved_tensors
        return _ln_backward(dy.contiguous(), x, scale, cu, mean, rstd, ctx.eps) + (None, None, None)


def ln_modulate(x, shift, scale, eps=1e-6, cu_seqlens=None, save_stats=True):
    """y = LayerNorm(x) * (1 + scale) + shift (no affine, fp32 statistics).  save_stats=False keeps
    only x between the passes; the backward then recomputes mean and rstd."""
    host = lnmod.native()
    y = None if host is None else host.ln_modulate(x, shift, scale, cu_seqlens, float(eps), bool(save_stats))
    return _LnModulate.apply(x, shift, scale, cu_seqlens, float(eps), bool(save_stats)) if y is None else y


def _gated_backward(dy, dh, h, u, gate, scale, mean, rstd, cu_seqlens, eps):
    return lnmod._gated_backward(dy, dh, h, u, gate, scale, mean, rstd, cu_seqlens, eps, io_grads=True)


class _GatedLnModulate(torch.autograd.Function):
    """Sec. 4.4 "Gate + Norm": the residual update and the LayerNorm-Modulate after it."""

    @staticmethod
    def forward(ctx, x, u, gate, shift, scale, cu_seqlens, eps):
        _contig(x, u, gate, shift, scale, cu_seqlens)
        h, y, mean, rstd = lnmod.gated_forward(x, u, gate, shift, scale, cu_seqlens, eps)
        ctx.eps = eps
        ctx.save_for_backward(h, u, gate, scale, cu_seqlens, mean, rstd)
        return h, y

    @staticmethod
    def backward(ctx, dh, dy):
        h, u, gate, scale, cu, mean, rstd = ctx.saved_tensors
        return _gated_backward(dy.contiguous(), dh.contiguous(), h, u, gate, scale, mean, rstd, cu,
                               ctx.eps) + (None, None)


def gated_ln_modulate(x, u, gate, shift, scale, eps=1e-6, cu_seqlens=None):
    """h = x + gate * u (returned, it is the new residual stream) and y = LN(h) * (1 + scale) + shift."""
    host = lnmod.native()
    r = None if host is None else host.gated_ln_modulate(x, u, gate, shift, scale, cu_seqlens, float(eps))
    return _GatedLnModulate.apply(x, u, gate, shift, scale, cu_seqlens, float(eps)) if r is None else r


def _qk_backward(dqn, dkn, q, k, wq, wk, rq, rk, eps):
    return lnmod._qknorm_backward(dqn, dkn, q, k, wq, wk, rq, rk, eps, io_grads=True)


class _QkNorm(torch.autograd.Function):
    """Sec. 4.4 fused Q-Norm + K-Norm."""

    @staticmethod
    def forward(ctx, q, k, wq, wk, eps):
        _contig(q, k, wq, wk)
        qn, kn, rq, rk = lnmod.qknorm_forward(q, k, wq, wk, eps)
        ctx.eps = eps
        ctx.save_for_backward(q, k, wq, wk, rq, rk)
        return qn, kn

    @staticmethod
    def backward(ctx, dqn, dkn):
        q, k, wq, wk, rq, rk = ctx.saved_tensors
        return _qk_backward(dqn.contiguous(), dkn.contiguous(), q, k, wq, wk, rq, rk, ctx.eps) + (None,)


def qk_norm(q, k, wq, wk, eps=1e-6):
    """q * rsqrt(mean(q^2) + eps) * wq and the same for k, in one launch."""
    host = lnmod.native()
    r = None if host is None else host.qk_norm(q, k, wq, wk, float(eps))
    return _QkNorm.apply(q, k, wq, wk, float(eps)) if r is None else r


def _ckpt_backward(dy, codes, scales, scale, mean, rstd, cu_seqlens, group):
    return lnmod._backward_ckpt(dy, codes, scales, scale, mean, rstd, cu_seqlens, int(group), io_grads=True)


class _LnModulateCkpt(torch.autograd.Function):
    """ln_modulate whose backward reads the 8-bit checkpoint that the forward wrote beside y."""

    @staticmethod
    def forward(ctx, x, shift, scale, cu_seqlens, eps, code, group):
        _contig(x, shift, scale, cu_seqlens)
        y, codes, scales, mean, rstd = lnmod.forward_ckpt(x, shift, scale, cu_seqlens, eps, code, group)
        ctx.group = group
        ctx.save_for_backward(codes, scales, scale, cu_seqlens, mean, rstd)
        return y

    @staticmethod
    def backward(ctx, dy):
        codes, scales, scale, cu, mean, rstd = ctx.saved_tensors
        return _ckpt_backward(dy.contiguous(), codes, scales, scale, mean, rstd, cu, ctx.group) + (None,) * 4


def ln_modulate_ckpt(x, shift, scale, eps=1e-6, cu_seqlens=None, code="int8", group=128):
    """ln_modulate that keeps x in 8 bits between the passes ("int8" or "e4m3", one scale for each `group` = 32, 64 or 128
    features of a row): D + 4 ceil(D / group) + 8 bytes per token where ln_modulate keeps 2 D + 8 (bf16).  y and dshift
    are ln_modulate's; dx and dscale are formed with the values that the codes stand for, at most half a code's step from
    x (int8: 1/254 of the group's largest value)."""
    host = lnmod.native()
    y = None if host is None else host.ln_modulate_ckpt(x, shift, scale, cu_seqlens, float(eps), code, group)
    return _LnModulateCkpt.apply(x, shift, scale, cu_seqlens, float(eps), code, group) if y is None else y


def _rms_quant_backward(dy, h, w, rstd, dh, own_dr):
    return lnmod._rmsnorm_quant_backward(dy, h, w, rstd, dh, io_grads=True, own_dr=bool(own_dr))


class _RmsNormQuant(torch.autograd.Function):
    """RMS norm of x (+ residual), rounded to 8 bits and back; the gradient passes straight through the rounding."""

    @staticmethod
    def forward(ctx, x, w, residual, eps, code, group):
        _contig(x, w, residual)
        _, _, y, h, rstd = lnmod._rmsnorm_quant(x, w, residual, eps, code, group)
        ctx.save_for_backward(h, w, rstd)
        ctx.residual = residual is not None
        return (h, y) if ctx.residual else y

    @staticmethod
    def backward(ctx, *grads):
        h, w, rstd = ctx.saved_tensors
        dh = grads[0].contiguous() if ctx.residual else None
        both = ctx.residual and ctx.needs_input_grad[0] and ctx.needs_input_grad[2]
        dx, dw, dr = _rms_quant_backward(grads[-1].contiguous(), h, w, rstd, dh, both)
        return dx, dw, dr if ctx.residual else None, None, None, None


def rms_norm_quant(x, w, residual=None, eps=1e-6, code="e4m3", group=0):
    """y = h * rsqrt(mean(h^2) + eps) * w rounded to 8 bits (one scale for each `group` = 32, 64 or 128 features, or 0: for
    a row), as the values that the codes stand for: what a model trains on that is served with lnmod.rmsnorm_quant_forward.
    h = x; with a residual h = x + residual, and (h, y) is returned."""
    host = lnmod.native()
    r = None if host is None else host.rms_norm_quant(x, w, residual, float(eps), code, group)
    return _RmsNormQuant.apply(x, w, residual, float(eps), code, group) if r is None else r


def _readable(t):
    """A gradient as the kernels can read it."""
    return t if t.layout == torch.strided and lnmod._heads_strides(t) is not None else t.contiguous()


def _rotary_backward(dq, dk, positions, table, axes, interleaved):
    return lnmod.rotary(_readable(dq), None if dk is None else _readable(dk), positions, table, tuple(axes), bool(interleaved),
                        inverse=True)


class _Rotary(torch.autograd.Function):
    """The rotation; its gradient is the rotation backwards."""

    @staticmethod
    def forward(ctx, q, k, positions, table, axes, interleaved):
        qr, kr = lnmod.rotary(q, k, positions, table, axes, interleaved)
        ctx.save_for_backward(positions, table)
        ctx.axes, ctx.interleaved = axes, interleaved
        return qr if k is None else (qr, kr)

    @staticmethod
    def backward(ctx, dq, dk=None):
        positions, table = ctx.saved_tensors
        return _rotary_backward(dq, dk, positions, table, ctx.axes, ctx.interleaved) + (None,) * 4


def rotary(q, k, positions, table, axes, interleaved=True):
    """Rotary positions with several axes of q and k, [B, S, heads, head_dim] or packed [T, heads, head_dim]; k may be None,
    and one tensor is returned then; the table gets no gradient.  See lnmod.rotary, lnmod.rotary_table and lnmod.rotary_grid."""
    host = lnmod.native()
    r = None if host is None else host.rotary(q, k, positions, table, axes, interleaved)
    return _Rotary.apply(q, k, positions, table, axes, interleaved) if r is None else r


def _qk_rotary_backward(dqr, dkr, q, k, wq, wk, rq, rk, positions, table, axes, interleaved):
    return lnmod._qknorm_rotary_backward(_readable(dqr), _readable(dkr), q, k, wq, wk, rq, rk, positions, table, tuple(axes),
                                         bool(interleaved), io_grads=True)


class _QkNormRotary(torch.autograd.Function):
    """Q-Norm + K-Norm and the rotation."""

    @staticmethod
    def forward(ctx, q, k, wq, wk, positions, table, axes, interleaved, eps):
        qr, kr, rq, rk = lnmod.qknorm_rotary_forward(q, k, wq, wk, positions, table, axes, interleaved, eps)
        ctx.save_for_backward(q, k, wq, wk, rq, rk, positions, table)
        ctx.axes, ctx.interleaved = axes, interleaved
        return qr, kr

    @staticmethod
    def backward(ctx, dqr, dkr):
        q, k, wq, wk, rq, rk, positions, table = ctx.saved_tensors
        return _qk_rotary_backward(dqr, dkr, q, k, wq, wk, rq, rk, positions, table, ctx.axes, ctx.interleaved) + (None,) * 5


def qk_norm_rotary(q, k, wq, wk, positions, table, axes, interleaved=True, eps=1e-6):
    """rotary(qk_norm(...)) in one pass, rounded once.  wq, wk: [heads * head_dim] of each tensor (the norm is over a token's
    whole row), or both [head_dim] (over each head)."""
    host = lnmod.native()
    r = None if host is None else host.qk_norm_rotary(q, k, wq, wk, positions, table, axes, interleaved, float(eps))
    return _QkNormRotary.apply(q, k, wq, wk, positions, table, axes, interleaved, float(eps)) if r is None else r
