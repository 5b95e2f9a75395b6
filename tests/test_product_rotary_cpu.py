"""What row codes, their product and the rotations refuse, checked without a GPU: the C entry points validate before any HIP
call, the Python wrappers look at shape, element type and layout before the device."""
import ctypes
import math

import pytest
import torch

from paper_2605_17923_amd import functional, lnmod

A = 0x1000          # a 16-byte aligned fake address; validation never dereferences it
EINVAL, EUNS, EALIGN, EWS, OK = (lnmod.LNMOD_EINVAL, lnmod.LNMOD_EUNSUPPORTED, lnmod.LNMOD_EALIGN, lnmod.LNMOD_EWORKSPACE,
                                 lnmod.LNMOD_OK)
bf, f32, i32, i8 = torch.bfloat16, torch.float32, torch.int32, torch.int8


def rows(x=A, N=4, D=64, codes=A, s=A, dtype=0, code=0):
    return lnmod.lnmod_quantize_rows(x, N, D, None, codes, s, dtype, code)


def test_row_codes_rejections():
    for name in ("x", "codes", "s"):
        assert rows(**{name: None}) == EINVAL
    assert rows(N=-1) == EINVAL and rows(N=1 << 31) == EINVAL and rows(dtype=2) == EINVAL and rows(code=2) == EINVAL
    assert rows(D=0) == EUNS and rows(D=60) == EUNS and rows(D=60, dtype=1) == EUNS and rows(D=(1 << 20) + 8) == EUNS
    assert rows(x=A + 8) == EALIGN and rows(codes=A + 8) == EALIGN
    assert rows(N=0) == OK and rows(N=0, x=None) == OK


def product(a=A, sa=A, w=A, sw=A, bias=None, M=4, N=5, K=64, y=A, dtype=0, code=0):
    return lnmod.lnmod_code_product(a, sa, w, sw, bias, M, N, K, None, y, dtype, code)


def test_product_rejections():
    for name in ("a", "sa", "w", "sw", "y"):
        assert product(**{name: None}) == EINVAL, name
    for name in ("a", "w", "y"):
        assert product(**{name: A + 8}) == EALIGN, name
    for name in ("M", "N"):
        assert product(**{name: -1}) == EINVAL and product(**{name: 1 << 31}) == EINVAL, name
        assert product(**{name: 0}) == OK and product(**{name: 0}, a=None) == OK
    assert product(K=-8) == EINVAL and product(dtype=2) == EINVAL and product(code=2) == EINVAL and product(code=-1) == EINVAL
    assert product(K=0) == EUNS and product(K=60) == EUNS and product(K=4) == EUNS and product(K=1 << 17) == EUNS


def heads(data=A, batch=64, token=64, head=16):
    return lnmod.Heads(data, batch, token, head)


def rot(pos=A, rows=4, table=A, table_rows=9, axes=(8, 4, 4), interleaved=1, n=None):
    f = (ctypes.c_int32 * 4)(*axes[:4])
    return lnmod.Rotation(pos, rows, table, table_rows, len(axes) if n is None else n, f, interleaved)


def rotary(q="q", k="k", B=2, S=4, hq=4, hk=4, hd=16, r=None, qo=A, ko=A, dtype=0):
    q = heads() if q == "q" else q
    k = heads() if k == "k" else k
    return lnmod.lnmod_rotary(q, k, B, S, hq, hk, hd, rot() if r is None else r, 0, None, qo, ko, dtype)


def fwd(q="q", k="k", wq=A, wk=A, B=2, S=4, hq=4, hk=4, hd=16, r=None, eps=1e-6, per_head=0, qo=A, ko=A, rq=A, rk=A, dtype=0):
    q = heads() if q == "q" else q
    k = heads() if k == "k" else k
    return lnmod.lnmod_qknorm_rotary_forward(q, k, wq, wk, B, S, hq, hk, hd, rot() if r is None else r, eps, per_head, None, qo,
                                             ko, rq, rk, dtype)


def bwd(dqo="q", dko="k", q="q", k="k", wq=A, wk=A, B=2, S=4, hq=4, hk=4, hd=16, r=None, per_head=0, rq=A, rk=A, dq=A, dk=A,
        dwq=A, dwk=A, ws=A, ws_bytes=1 << 40, dtype=0, io=0):
    dqo, dko, q, k = (heads() if t in ("q", "k") else t for t in (dqo, dko, q, k))
    return lnmod.lnmod_qknorm_rotary_backward(dqo, dko, q, k, wq, wk, B, S, hq, hk, hd, rot() if r is None else r, per_head, None,
                                              rq, rk, dq, dk, dwq, dwk, ws, ws_bytes, dtype, io)


@pytest.mark.parametrize("call", [rotary, fwd, bwd])
def test_rotation_rejections(call):
    assert call(q=None) == EINVAL and call(q=heads(None)) == EINVAL and call(k=heads(None)) == EINVAL
    assert call(q=heads(A + 8)) == EALIGN and call(k=heads(token=68)) == EALIGN and call(q=heads(head=4)) == EALIGN
    assert call(q=heads(batch=-64)) == EINVAL and call(dtype=2) == EINVAL
    assert call(B=-1) == EINVAL and call(S=-1) == EINVAL and call(B=1 << 16, S=1 << 15) == EINVAL
    assert call(hq=0) == EINVAL and call(hq=-1) == EINVAL and call(hk=-1) == EINVAL
    for hd in (0, 4, 12, 264):
        assert call(hd=hd) == EUNS
    assert call(hq=(1 << 16) + 1) == EUNS
    assert call(r=rot(axes=(8, 4, 6))) == EUNS                                  # more features than a head has
    assert call(r=rot(axes=(8, 3, 3))) == EUNS and call(r=rot(axes=(8, 0, 8))) == EUNS
    assert call(r=rot(axes=(6, 4, 4), interleaved=0)) == EUNS                   # halves: a multiple of 8 in all
    assert call(r=rot(n=0)) == EINVAL and call(r=rot(n=5)) == EINVAL and call(r=rot(axes=(8, -4, 4))) == EINVAL
    assert call(r=rot(pos=None)) == EINVAL and call(r=rot(table=None)) == EINVAL and call(r=rot(table_rows=0)) == EINVAL
    assert call(r=rot(rows=5)) == EINVAL and call(r=rot(table=A + 4)) == EALIGN
    assert call(r=rot(table_rows=1 << 31)) == EINVAL


def test_rotary_rejections():
    assert rotary(k=None) == EINVAL and rotary(ko=None) == EINVAL and rotary(hk=0) == EINVAL and rotary(qo=None) == EINVAL
    assert rotary(qo=A + 8) == EALIGN and rotary(ko=A + 8) == EALIGN
    assert rotary(S=0) == OK and rotary(B=0, r=rot(pos=None)) == OK


def test_no_tokens_need_no_addresses():
    for B, S in ((1, 0), (0, 5), (2, 0)):
        none = dict(B=B, S=S, q=heads(None), k=heads(None), r=rot(pos=None, rows=0), qo=None, ko=None)
        assert rotary(**none) == OK and rotary(**none, dtype=1) == OK
        assert fwd(**none, wq=None, wk=None, rq=None, rk=None) == OK
        assert rotary(**{**none, "r": rot(axes=(8, 4, 6))}) == EUNS
    assert rotary(ko=None) == EINVAL and rotary(k=None, hk=0) == EINVAL


def test_norm_with_rotation_rejections():
    for call, names in ((fwd, ("wq", "wk", "qo", "ko", "rq", "rk")), (bwd, ("wq", "wk", "dq", "dk", "rq", "rk", "dwq", "dwk"))):
        for name in names:
            assert call(**{name: None}) == EINVAL, name
            if not name.startswith(("r", "dw")):
                assert call(**{name: A + 8}) == EALIGN, name
        assert call(k=None) == EINVAL and call(hk=0) == EINVAL
        assert call(hq=513) == EUNS and call(hk=513) == EUNS                    # 513 * 16 features in one row's norm
    assert fwd(eps=0.0) == EINVAL and fwd(eps=math.nan) == EINVAL and fwd(S=0) == OK and fwd(S=0, qo=None) == OK
    assert bwd(dqo=None) == EINVAL and bwd(dko=heads(A, 60, 64, 16)) == EALIGN
    assert bwd(dwq=A + 4, io=1) == EALIGN and bwd(S=0, dwq=None) == EINVAL
    need = lnmod.lnmod_qknorm_rotary_backward_workspace_bytes(8, 4, 4, 16, 0)
    assert need > 0 and bwd(ws=None) == EWS and bwd(ws_bytes=need - 1) == EWS and bwd(ws=A + 4, ws_bytes=need) == EALIGN
    for bad in ((-1, 4, 4, 16, 0), (1 << 31, 4, 4, 16, 0), (8, 0, 4, 16, 0), (8, 4, 4, 12, 0), (8, 513, 4, 16, 0), (8, 4, 4, 264, 1)):
        assert lnmod.lnmod_qknorm_rotary_backward_workspace_bytes(*bad) == 0


@pytest.mark.parametrize("per_head", [0, 1])
@pytest.mark.parametrize("shape", [(40, 40, 128), (24, 8, 96), (1, 1, 8), (12, 4, 64), (31, 7, 136), (32, 32, 256)])
def test_workspace_never_falls_as_the_tokens_grow(shape, per_head):
    last = 0
    for n in list(range(0, 700)) + [1 << k for k in range(10, 31)]:
        size = lnmod.lnmod_qknorm_rotary_backward_workspace_bytes(n, *shape, per_head)
        assert size >= last
        last = size


def t(*shape, dtype=bf):
    return torch.zeros(*shape, dtype=dtype)


def rejects(fn, *args, match=None, **kw):
    with pytest.raises(ValueError, match=match):
        fn(*args, **kw)


def test_product_wrapper_rejections():
    x = t(3, 4, 64)
    rejects(lnmod.quantize_rows, x, "int4", match="int8")
    rejects(lnmod.quantize_rows, x.half(), match="bfloat16 or float32")
    rejects(lnmod.quantize_rows, x.transpose(0, 1), match="contiguous")
    rejects(lnmod.quantize_rows, torch.tensor(1.0), match="D")
    rejects(lnmod.quantize_rows, x, match="GPU")
    c, s, w, sw = t(3, 4, 64, dtype=i8), t(3, 4, dtype=f32), t(5, 64, dtype=i8), t(5, dtype=f32)
    rejects(lnmod.code_product, x, s, w, sw, match="int8 or float8")
    rejects(lnmod.code_product, c, t(3, 4, 1, dtype=f32), w, sw, match="scales must have shape")
    rejects(lnmod.code_product, c, s, t(5, 72, dtype=i8), sw, match="w must have shape")
    rejects(lnmod.code_product, c, s, w.to(torch.float8_e4m3fn), sw, match="w must be")
    rejects(lnmod.code_product, c, s, t(64, 5, dtype=i8).t(), sw, match="contiguous")
    rejects(lnmod.code_product, c, s, w[0], sw, match=r"\[N, K\]")
    rejects(lnmod.code_product, c, s, w, sw[:4], match="w_scales must have shape")
    rejects(lnmod.code_product, c, s, w, sw, t(5, dtype=f32), match="bias must be")
    rejects(lnmod.code_product, c, s, w, sw, t(4), match="bias must have shape")
    rejects(lnmod.code_product, c, s, w, sw, None, torch.float16, match="dtype")
    rejects(lnmod.code_product, c, s, w, sw, match="GPU")


def test_rotary_wrapper_rejections():
    q, k, pos, table, axes = t(2, 6, 4, 16), t(2, 6, 2, 16), t(6, 3, dtype=i32), t(9, 8, 2, dtype=f32), (8, 4, 4)
    wq, wk = t(16), t(16)
    for fn, w in ((functional.rotary, ()), (lnmod.rotary, ()), (functional.qk_norm_rotary, (wq, wk)), (lnmod.qknorm_rotary_forward, (wq, wk))):
        rejects(fn, q[0, 0], k, *w, pos, table, axes, match="head_dim")
        rejects(fn, q.half(), k, *w, pos, table, axes, match="bfloat16 or float32")
        rejects(fn, q, k[:1], *w, pos, table, axes, match="k must have shape")
        rejects(fn, q, k.float(), *w, pos, table, axes, match="k must be")
        rejects(fn, t(2, 6, 4, 32)[..., ::2], k, *w, pos, table, axes, match="dense features")
        rejects(fn, t(2, 6, 4, 20)[..., :16], k, *w, pos, table, axes, match="16-byte")
        rejects(fn, q, k, *w, pos.long(), table, axes, match="positions must be")
        rejects(fn, q, k, *w, pos[:5], table, axes, match="positions must have shape")
        rejects(fn, q, k, *w, t(1, 6, 3, dtype=i32), table, axes, match="positions must have shape")
        rejects(fn, q, k, *w, pos, table[:, :7], axes, match="table must have shape")
        rejects(fn, q, k, *w, pos, table.double(), axes, match="table must be")
        rejects(fn, q, k, *w, pos, table[:0], axes, match="a position")
        for bad in ((8, 4, 3), (), (16, 0), (2,) * 5, 16, (8.0, 8.0), None):
            rejects(fn, q, k, *w, pos, table, bad, match="axes")
        rejects(fn, q, k, *w, pos, t(9, 12, 2, dtype=f32), (8, 8, 8), match="a head has 16")
        rejects(fn, q, k, *w, pos, t(9, 7, 2, dtype=f32), (6, 4, 4), False, match="multiple of 8")
        rejects(fn, q, k, *w, pos, table, axes, 1, match="interleaved")
        rejects(fn, q, k, *w, pos, table, axes, match="GPU")
    for fn in (functional.qk_norm_rotary, lnmod.qknorm_rotary_forward):
        rejects(fn, q, None, wq, wk, pos, table, axes, match="k must be")
        rejects(fn, q, k, t(64), wk, pos, table, axes, match="wk must have shape")
        rejects(fn, q, k, wq, t(32), pos, table, axes, match="wq must have shape")
        rejects(fn, q, k, wq.float(), wk, pos, table, axes, match="wq must be")
    r, rk = t(2, 6, 4, dtype=f32), t(2, 6, 2, dtype=f32)
    rejects(lnmod.qknorm_rotary_backward, q[:1], k, q, k, wq, wk, r, rk, pos, table, axes, match="dq_out must have shape")
    rejects(lnmod.qknorm_rotary_backward, q, k, q, k, wq, wk, r[..., 0], rk, pos, table, axes, match="rstd_q must have shape")
    rejects(lnmod.qknorm_rotary_backward, q, k, q, k, wq, wk, r, rk, pos, table, axes, ws=torch.zeros(8, dtype=torch.uint8), match="bytes")
    rejects(lnmod.qknorm_rotary_backward, q, k, q, k, wq, wk, r, rk, pos, table, axes, match="GPU")


def test_tables_and_grids():
    table = lnmod.rotary_table(5, (4, 2), base=100.0, device="cpu")
    assert table.shape == (5, 3, 2) and table.dtype == f32
    for p in range(5):
        for j, f in enumerate((1.0, 0.1, 1.0)):
            assert abs(float(table[p, j, 0]) - math.cos(p * f)) <= 2.0 ** -24 and abs(float(table[p, j, 1]) - math.sin(p * f)) <= 2.0 ** -24
    shifted = lnmod.rotary_table([-2, 0.5], (4,), frequencies=[1.0, 3.0], device="cpu")
    assert abs(float(shifted[0, 1, 1]) - math.sin(-6.0)) <= 2.0 ** -24 and abs(float(shifted[1, 0, 0]) - math.cos(0.5)) <= 2.0 ** -24
    rejects(lnmod.rotary_table, 4, (4, 4), frequencies=[1.0], match="frequencies")
    rejects(lnmod.rotary_table, [[1.0]], (4,), match="positions")
    grid = lnmod.rotary_grid(2, 3, 4, device="cpu")
    assert grid.dtype == i32 and grid.shape == (24, 3) and grid[5].tolist() == [0, 1, 1] and grid[-1].tolist() == [1, 2, 3]
