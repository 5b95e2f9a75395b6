"""What the form of the norm's backward with two gradients refuses; the C entry points validate before any HIP call."""
from paper_2605_17923_amd import lnmod

A = 0x1000          # a 16-byte aligned fake address; validation never dereferences it


def call(dy=A, dh=A, h=A, w=A, N=4, D=64, rstd=A, dx=A, dr=A, dw=A, ws=A, ws_bytes=1 << 40, dtype=0, io=0):
    return lnmod.lnmod_rmsnorm_quant_backward_residual(dy, dh, h, w, N, D, None, rstd, dx, dr, dw, ws, ws_bytes, dtype, io)


def test_rejections():
    for name in ("dy", "h", "w", "rstd", "dx", "dr", "dw"):
        assert call(**{name: None}) == lnmod.LNMOD_EINVAL, name
    for name in ("dy", "dh", "h", "w", "dx", "dr"):
        assert call(**{name: A + 8}) == lnmod.LNMOD_EALIGN, name
    assert call(N=-1) == lnmod.LNMOD_EINVAL and call(N=1 << 31) == lnmod.LNMOD_EINVAL and call(dtype=2) == lnmod.LNMOD_EINVAL
    assert call(D=60, dtype=1) == lnmod.LNMOD_EUNSUPPORTED and call(D=8200) == lnmod.LNMOD_EUNSUPPORTED
    need = lnmod.lnmod_rmsnorm_quant_backward_workspace_bytes(4, 64)
    assert call(ws=None) == lnmod.LNMOD_EWORKSPACE and call(ws_bytes=need - 1) == lnmod.LNMOD_EWORKSPACE
    assert call(ws=A + 4, ws_bytes=need) == lnmod.LNMOD_EALIGN and call(dw=A + 8, io=1) == lnmod.LNMOD_EALIGN
