"""What the 8-bit operators refuse, checked without a GPU: the C entry points validate before any HIP call, the Python
wrappers look at shape, element type and layout before the device."""
import pytest
import torch

from paper_2605_17923_amd import functional, lnmod

A = 0x1000          # a 16-byte aligned fake address; validation never dereferences it
EINVAL, EUNS, EALIGN, EWS, OK = (lnmod.LNMOD_EINVAL, lnmod.LNMOD_EUNSUPPORTED, lnmod.LNMOD_EALIGN, lnmod.LNMOD_EWORKSPACE,
                                 lnmod.LNMOD_OK)
bf, f32 = torch.bfloat16, torch.float32


def quantize(x=A, N=4, D=64, group=32, codes=A, s=A, dtype=0, code=0):
    return lnmod.lnmod_quantize(x, N, D, group, None, codes, s, dtype, code)


def dequantize(x=A, N=4, D=64, group=32, codes=A, s=A, dtype=0, code=0):
    return lnmod.lnmod_dequantize(codes, s, N, D, group, None, x, dtype, code)


@pytest.mark.parametrize("call", [quantize, dequantize])
def test_checkpoint_rejections(call):
    for name in ("x", "codes", "s"):
        assert call(**{name: None}) == EINVAL
    assert call(N=-1) == EINVAL and call(N=1 << 31) == EINVAL and call(D=-8) == EINVAL
    assert call(group=16) == EINVAL and call(group=256) == EINVAL and call(group=-32) == EINVAL
    assert call(dtype=2) == EINVAL and call(code=2) == EINVAL and call(code=-1) == EINVAL
    assert call(D=0) == EUNS and call(D=60) == EUNS and call(D=60, dtype=1) == EUNS and call(D=(1 << 20) + 8) == EUNS
    assert call(x=A + 8) == EALIGN and call(codes=A + 8) == EALIGN
    assert call(N=0) == OK and call(N=0, x=None) == OK


def test_a_scale_for_a_whole_row_is_read_but_not_written():
    assert quantize(group=0) == EINVAL
    assert dequantize(group=0, x=None) == EINVAL and dequantize(group=0, x=A + 4) == EALIGN


def fwd(x=A, shift=A, scale=A, cu=None, n=2, s=4, D=64, eps=1e-6, group=32, y=A, codes=A, cs=A, mean=A, rstd=A, dtype=0,
        mod=0, code=0):
    return lnmod.lnmod_forward_ckpt(x, shift, scale, cu, n, s, D, eps, group, None, y, codes, cs, mean, rstd, dtype, mod, code)


def bwd(dy=A, codes=A, cs=A, scale=A, cu=None, n=2, s=4, D=64, group=32, mean=A, rstd=A, dx=A, dshift=A, dscale=A, ws=A,
        ws_bytes=1 << 40, dtype=0, mod=0, code=0, io=0):
    return lnmod.lnmod_backward_ckpt(dy, codes, cs, scale, cu, n, s, D, group, None, mean, rstd, dx, dshift, dscale, ws,
                                     ws_bytes, dtype, mod, code, io)


def test_forward_ckpt_rejections():
    for name in ("x", "shift", "scale", "y", "codes", "cs", "mean", "rstd"):
        assert fwd(**{name: None}) == EINVAL, name
    for name in ("x", "shift", "scale", "y", "codes"):
        assert fwd(**{name: A + 8}) == EALIGN, name
    assert fwd(n=-1) == EINVAL and fwd(s=-1) == EINVAL and fwd(n=1 << 20, s=1 << 20) == EINVAL
    assert fwd(eps=0.0) == EINVAL and fwd(eps=float("nan")) == EINVAL
    assert fwd(group=0) == EINVAL and fwd(group=48) == EINVAL and fwd(code=2) == EINVAL
    assert fwd(dtype=2) == EINVAL and fwd(mod=2) == EINVAL
    assert fwd(cu=A, mod=1) == EINVAL                                    # packed batches: one row per segment
    assert fwd(cu=A, n=0) == EINVAL                                      # tokens that belong to no segment
    assert fwd(D=60) == EUNS and fwd(D=60, dtype=1) == EUNS and fwd(D=8200) == EUNS and fwd(D=0) == EUNS
    assert fwd(n=0) == OK and fwd(s=0) == OK and fwd(s=0, x=None) == OK and fwd(cu=A, n=0, s=0) == OK


def test_backward_ckpt_rejections():
    for name in ("dy", "codes", "cs", "scale", "mean", "rstd", "dx", "dshift", "dscale"):
        assert bwd(**{name: None}) == EINVAL, name
        assert bwd(**{name: None}, mod=1, ws=None, ws_bytes=0) == EINVAL, name
    for name in ("dy", "codes", "scale", "dx", "dshift", "dscale"):
        assert bwd(**{name: A + 8}) == EALIGN, name
    assert bwd(cu=A, mod=1) == EINVAL and bwd(group=16) == EINVAL and bwd(code=7) == EINVAL and bwd(mod=-1) == EINVAL
    assert bwd(D=60, dtype=1) == EUNS and bwd(D=8200) == EUNS
    assert bwd(ws=None) == EWS
    need = lnmod.lnmod_backward_ckpt_workspace_bytes(2, 8, 64)
    assert need > 0 and bwd(ws_bytes=need - 1) == EWS and bwd(ws=A + 4, ws_bytes=need) == EALIGN
    assert bwd(n=0) == OK and bwd(s=0, mod=1) == OK
    assert bwd(s=0, dshift=None) == EINVAL and bwd(s=0, dscale=A + 2) == EALIGN
    for bad in ((-1, 8, 64), (1, -1, 64), (1, 1 << 31, 64), (1, 8, 60), (1, 8, 8200), (1, 8, 0)):
        assert lnmod.lnmod_backward_ckpt_workspace_bytes(*bad) == 0


def rms(x=A, r=A, w=A, N=4, D=64, eps=1e-6, group=0, h=A, codes=A, cs=A, y=None, rstd=A, dtype=0, code=1):
    return lnmod.lnmod_rmsnorm_quant_forward(x, r, w, N, D, eps, group, None, h, codes, cs, y, rstd, dtype, code)


def rmsb(dy=A, dh=A, h=A, w=A, N=4, D=64, rstd=A, dx=A, dw=A, ws=A, ws_bytes=1 << 40, dtype=0, io=0):
    return lnmod.lnmod_rmsnorm_quant_backward(dy, dh, h, w, N, D, None, rstd, dx, dw, ws, ws_bytes, dtype, io)


def test_rmsnorm_quant_rejections():
    for name in ("x", "w", "rstd", "codes", "cs", "r", "h"):             # r without h, codes without scales
        assert rms(**{name: None}) == EINVAL, name
    assert rms(y=A) == EINVAL and rms(codes=None, cs=None) == EINVAL     # exactly one output
    assert rms(codes=None, y=A) == EINVAL                                # scales without codes
    for name in ("x", "r", "w", "h", "codes"):
        assert rms(**{name: A + 8}) == EALIGN, name
    assert rms(codes=None, cs=None, y=A + 8) == EALIGN
    assert rms(group=16) == EINVAL and rms(code=2) == EINVAL and rms(dtype=3) == EINVAL and rms(eps=-1.0) == EINVAL
    assert rms(N=-1) == EINVAL and rms(N=1 << 31) == EINVAL
    assert rms(D=60, dtype=1) == EUNS and rms(D=8200) == EUNS and rms(D=4) == EUNS
    assert rms(N=0) == OK and rms(N=0, x=None) == OK
    for name in ("dy", "h", "w", "rstd", "dx", "dw"):
        assert rmsb(**{name: None}) == EINVAL, name
    for name in ("dy", "dh", "h", "w", "dx"):
        assert rmsb(**{name: A + 8}) == EALIGN, name
    assert rmsb(dw=A + 8, io=1) == EALIGN and rmsb(dw=A + 4, ws=None) == EWS
    need = lnmod.lnmod_rmsnorm_quant_backward_workspace_bytes(4, 64)
    assert need > 0 and rmsb(ws_bytes=need - 1) == EWS and rmsb(ws=A + 4, ws_bytes=need) == EALIGN
    assert rmsb(N=-1) == EINVAL and rmsb(D=60, dtype=1) == EUNS and rmsb(dtype=2) == EINVAL and rmsb(N=0, dw=None) == EINVAL
    for bad in ((-1, 64), (1 << 31, 64), (8, 60), (8, 8200)):
        assert lnmod.lnmod_rmsnorm_quant_backward_workspace_bytes(*bad) == 0


def t(*shape, dtype=bf):
    return torch.zeros(*shape, dtype=dtype)


def rejects(fn, *args, match=None, **kw):
    with pytest.raises(ValueError, match=match):
        fn(*args, **kw)


def test_checkpoint_wrapper_rejections():
    x, c, s = t(3, 4, 64), t(3, 4, 64, dtype=torch.int8), t(3, 4, 2, dtype=f32)
    rejects(lnmod.quantize, x, "int4", match="int8")
    rejects(lnmod.quantize, x, 0, match="int8")
    for bad in (0, 16, 64.0, True, None):
        rejects(lnmod.quantize, x, "int8", bad, match="group")
    rejects(lnmod.quantize, t(3, 4, 64, dtype=torch.float16), match="bfloat16 or float32")
    rejects(lnmod.quantize, x.transpose(0, 1), match="contiguous")
    rejects(lnmod.quantize, torch.tensor(1.0), match="D")
    rejects(lnmod.quantize, x, "int8", 32, match="GPU")
    rejects(lnmod.dequantize, t(3, 4, 64, dtype=torch.uint8), s, bf, 32, match="int8 or float8")
    rejects(lnmod.dequantize, None, s, bf, 32, match="tensor")
    rejects(lnmod.dequantize, c, s, bf, 64, match="scales must have shape")
    rejects(lnmod.dequantize, c, s.double(), bf, 32, match="float32")
    rejects(lnmod.dequantize, c, s, bf, 0, match="scales must have shape")
    rejects(lnmod.dequantize, c, s, torch.float16, 32, match="dtype")
    rejects(lnmod.dequantize, c, s, "bf16", 32, match="dtype")
    rejects(lnmod.dequantize, c, s, bf, 32, match="GPU")
    rejects(lnmod.dequantize, c.to(torch.float8_e4m3fn), t(3, 4, dtype=f32), bf, 0, match="GPU")


def test_ckpt_wrapper_rejections():
    B, S, D = 2, 6, 64
    x, sh, sc = t(B, S, D), t(B, D), t(B, D)
    for fn in (lnmod.forward_ckpt, functional.ln_modulate_ckpt):
        rejects(fn, x, sh, t(B + 1, D), match="shape")
        rejects(fn, x, sh.float(), sc, match="shift must be")
        rejects(fn, t(B * S, D), sh, sc, match=r"\[B, S, D\]")
        rejects(fn, x, sh, sc, cu_seqlens=torch.tensor([0, 6, 12], dtype=torch.int32), match="packed")
        rejects(fn, x, sh, sc, code="fp8", match="int8")
        rejects(fn, x, sh, sc, group=0, match="group")
        rejects(fn, x, sh, sc, match="GPU")
    rejects(lnmod.forward_ckpt, t(B * S, D), sh, sc, torch.tensor([0, 6, 12]), match="int32")
    c, s, m = t(B, S, D, dtype=torch.int8), t(B, S, 1, dtype=f32), t(B, S, dtype=f32)
    rejects(lnmod.backward_ckpt, x, x, s, sc, m, m, match="int8 or float8")
    rejects(lnmod.backward_ckpt, x, c[:1], s, sc, m, m, match="codes must have shape")
    rejects(lnmod.backward_ckpt, x, c, s, sc, m, m, group=32, match="scales must have shape")
    rejects(lnmod.backward_ckpt, x, c, s, sc, m, None, match="rstd must be a tensor")
    rejects(lnmod.backward_ckpt, x, c, s, sc, m, m[:1], match="rstd must have shape")
    rejects(lnmod.backward_ckpt, x, c, s, sc, m, m, ws=torch.zeros(8, dtype=torch.uint8), match="bytes")
    rejects(lnmod.backward_ckpt, x, c, s, sc, m, m, match="GPU")


def test_rmsnorm_quant_wrapper_rejections():
    x, w = t(5, 64), t(64)
    for fn in (lnmod.rmsnorm_quant_forward, functional.rms_norm_quant):
        rejects(fn, x, t(72), match="w must have shape")
        rejects(fn, x, w.float(), match="w must be")
        rejects(fn, x, w, t(4, 64), match="residual must have shape")
        rejects(fn, x, w, t(64, 5).t(), match="contiguous")
        rejects(fn, x, w, code="e5m2", match="int8")
        rejects(fn, x, w, group=96, match="group")
        rejects(fn, x, w, x, match="GPU")
    r = t(5, dtype=f32)
    rejects(lnmod.rmsnorm_quant_backward, x, t(5, 72), w, r, match="w must have shape")
    rejects(lnmod.rmsnorm_quant_backward, t(4, 64), x, w, r, match="dy must have shape")
    rejects(lnmod.rmsnorm_quant_backward, x, x, w, r[:4], match="rstd must have shape")
    rejects(lnmod.rmsnorm_quant_backward, x, x, w, r, t(5, 64, dtype=f32), match="dh must be")
    rejects(lnmod.rmsnorm_quant_backward, x, x, w, r, ws=torch.zeros(8, dtype=torch.uint8), match="bytes")
    rejects(lnmod.rmsnorm_quant_backward, x, x, w, r, match="GPU")


def test_a_scale_for_a_row_needs_an_eps_that_bounds_rstd():
    call = lambda eps, group: lnmod.lnmod_rmsnorm_quant_forward(A, None, A, 0, 64, eps, group, None, None, A, A, None, A, 0, 0)   # noqa: E731
    assert call(1e-21, 0) == EUNS and call(1e-20, 0) == OK and call(1e-21, 32) == OK
