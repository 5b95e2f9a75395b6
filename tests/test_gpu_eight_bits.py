"""The operators that hold activations in 8 bits against the float64 oracle (oracle/code_oracle.py).

Tolerances.  Codes and scales of given values are functions of those values alone: they must be equal.  y, dx, dshift, dscale,
dw: as in the other parity tests (parity_util).  The codes of the normed rows: a code is the rounding of (h*rstd)*w / s, where
s goes with the same rstd, so six fp32 roundings lie between it and the exact quotient, 6 * 2^-24 < 4e-7 of it: the code
must lie between the codes of the exact quotient times 1 -+ 1e-6.  Its scale goes with rstd (1e-5, as in the other tests) and
three roundings: 1.1e-5."""
import numpy as np
import pytest
import torch

from oracle import code_oracle as co
from paper_2605_17923_amd import functional as F
from paper_2605_17923_amd import lnmod
from parity_util import check_f32_tensor, check_io_tensor, check_stats, to_host64

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
KIND = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    lnmod.library()
    yield
    torch.cuda.synchronize()


def make(seed, *shape, dtype="bf16", mean=0.0, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std + mean).to(DT[dtype]).cuda()


def acts(seed, *shape, dtype="bf16"):
    """Off centre, with rows of other sizes and one value in a hundred an outlier."""
    g = torch.Generator().manual_seed(seed)
    v = torch.randn(*shape, generator=g) * 2.0 + 0.5
    v *= torch.where(torch.rand(*shape, generator=g) < 1e-2, 20.0, 1.0)
    return v.to(DT[dtype]).cuda()


def bits(t):
    return t.view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


def same_bits(a, b):
    return a.dtype == b.dtype and a.shape == b.shape and torch.equal(bits(a), bits(b))


def expect_codes(codes, scales, v64, code, group):
    D = v64.shape[-1]
    want, s = co.encode(v64, code, group)
    assert codes.dtype == KIND[code] and scales.dtype == torch.float32
    got, gs = to_host64(codes).reshape(-1, D), to_host64(scales).reshape(s.shape)
    assert np.array_equal(np.isnan(gs), np.isnan(s)) and np.array_equal(gs[~np.isnan(s)], s[~np.isnan(s)])
    assert np.array_equal(got, want)
    return want, s


# ---- the checkpoint of a tensor ----------------------------------------------------------------------------------------
# widths: one unit, less than a group, whole groups, groups cut short, more than 64 units; N = 1, odd, more than the grid takes at once
@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,D,group", [(1, 8, 32), (3, 24, 128), (257, 32, 32), (5, 128, 64), (1001, 200, 32), (33, 264, 128),
                                       (70, 1432, 64), (129, 1536, 128), (9, 5120, 32), (3, 13824, 128), (2, 20488, 64),
                                       (40000, 40, 64), (30001, 512, 128)])
def test_quantize_and_back(N, D, group, dtype, code):
    print("case", N, D, group, dtype, code, flush=True)
    x = acts(N + D, N, D, dtype=dtype)
    x[0, : D // 2] = 0
    codes, scales = lnmod.quantize(x, code, group)
    assert codes.shape == x.shape and scales.shape == (N, -(-D // group))
    want, s = expect_codes(codes, scales, to_host64(x), code, group)
    back = lnmod.dequantize(codes, scales, x.dtype, group)
    exact = torch.from_numpy(co.decode(want, s, group))
    assert same_bits(back.cpu(), exact.float().to(x.dtype))               # one fp32 product, one rounding
    other = torch.float32 if dtype == "bf16" else torch.bfloat16
    assert same_bits(lnmod.dequantize(codes, scales, other, group).cpu(), exact.float().to(other))


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_at_the_ends_of_the_range(dtype, code):
    x = make(1, 12, 96, dtype=dtype)
    big = float(torch.finfo(DT[dtype]).max)
    x[0] = 0
    x[1, :32] = 2.0 ** -120
    x[2, 40] = float("inf")
    x[3, 41] = float("-inf")
    x[4, 42] = float("nan")
    x[5, 0], x[5, 1] = big, -big
    x[6, :32] = 2.0 ** -133                                               # below the normal numbers
    x[7] = -0.0
    x[8, 64:] = 2.0 ** -100
    x[9] = 1.0
    x[10, 0] = big
    x[11, 95] = float("nan")
    codes, scales = lnmod.quantize(x, code, 32)
    expect_codes(codes, scales, to_host64(x), code, 32)
    back = lnmod.dequantize(codes, scales, x.dtype, 32)
    nan = torch.zeros(12, 96, dtype=torch.bool)
    for row in (2, 3, 4):
        nan[row, 32:64] = True
    nan[11, 64:] = True
    assert torch.equal(back.isnan().cpu(), nan)


def test_every_largest_value():
    """Every significand that the largest value of a group can have: scale and codes as the correctly rounded quotients give
    them (in float64 on the device)."""
    n = 1 << 23
    x = torch.empty(n, 32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(5)
    x.uniform_(-1.0, 1.0, generator=g)
    x[:, 7] = (torch.arange(n, device="cuda", dtype=torch.int32) + 0x3f800000).view(torch.float32)
    for code, Q in (("int8", 127.0), ("e4m3", 448.0)):
        codes, scales = lnmod.quantize(x, code, 32)
        for part in range(0, n, 1 << 21):
            rows = slice(part, part + (1 << 21))
            s = (x[rows, 7].double() / torch.full((1,), Q, device="cuda", dtype=torch.float64)).float()
            assert torch.equal(scales[rows, 0], s)
            r = (1.0 / s.double()).float()
            p = x[rows].double() * r.double()[:, None]
            want = p.round() if code == "int8" else p.float().to(torch.float8_e4m3fn).double()
            assert torch.equal(codes[rows].double(), want)


def test_empty_tensors():
    for shape in ((0, 64), (3, 0, 64)):
        x = torch.empty(shape, device="cuda", dtype=torch.bfloat16)
        codes, scales = lnmod.quantize(x, "int8", 32)
        assert codes.shape == x.shape and scales.shape == shape[:-1] + (2,)
        assert lnmod.dequantize(codes, scales, torch.float32, 32).shape == x.shape
    w = make(2, 64)
    codes, scales, h, rstd = lnmod.rmsnorm_quant_forward(x, w)
    dx, dw = lnmod.rmsnorm_quant_backward(x, h, w, rstd)
    assert dx.shape == x.shape and not dw.any() and rstd.numel() == 0
    sh = torch.ones(3, 64, device="cuda", dtype=torch.bfloat16)
    y, codes, scales, mean, rstd = lnmod.forward_ckpt(x, sh, sh)
    dx, dsh, dsc = lnmod.backward_ckpt(x, codes, scales, sh, mean, rstd)
    assert y.shape == x.shape and not dsh.any() and not dsc.any() and dsh.shape == (3, 64)


# ---- LayerNorm-Modulate from a checkpoint ---------------------------------------------------------------------------------
def _batch(lens, B, S):
    """(row of the modulation tensor of each token, samples or segments, cu_seqlens or None)."""
    if lens is None:
        return np.repeat(np.arange(B), S), B, None
    cu = torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device="cuda")
    return np.repeat(np.arange(len(lens)), lens), len(lens), cu


def run_ckpt(D, dtype, code, group, lens=None, B=1, S=1, token=False, seed=7):
    print("ckpt case", D, dtype, code, group, lens if lens is None else len(lens), B, S, token, flush=True)
    of, n, cu = _batch(lens, B, S)
    T = len(of)
    shape = (T, D) if lens is not None else (B, S, D)
    mshape = shape if token else (n, D)
    x, dy = acts(seed, *shape, dtype=dtype), make(seed + 1, *shape, dtype=dtype)
    shift, scale = (make(seed + k, *mshape, dtype=dtype, std=0.2) for k in (2, 3))
    y, codes, scales, mean, rstd = lnmod.forward_ckpt(x, shift, scale, cu, 1e-6, code, group)
    assert codes.shape == x.shape and mean.shape == shape[:-1]
    plain_codes, plain_scales = lnmod.quantize(x, code, group)
    assert same_bits(codes, plain_codes) and same_bits(scales, plain_scales)
    x64, dy64 = to_host64(x).reshape(T, D), to_host64(dy).reshape(T, D)
    q, s = expect_codes(codes, scales, x64, code, group)
    if token:
        of = np.arange(T)
    sh64, sc64 = to_host64(shift).reshape(-1, D), to_host64(scale).reshape(-1, D)
    y64, mean64, rstd64 = co.ln_forward(x64, sh64, sc64, of, 1e-6)
    check_io_tensor("y", y, y64, dtype)
    check_stats(mean, rstd, mean64, rstd64)
    dx, dshift, dscale = lnmod.backward_ckpt(dy, codes, scales, scale, mean, rstd, cu, group)
    dx64, dsh64, dsc64 = co.ln_backward(dy64, co.decode(q, s, group), sc64, of, mean64, rstd64)
    check_io_tensor("dx", dx, dx64, dtype)
    if token:
        assert same_bits(dshift, dy)
        check_io_tensor("dscale", dscale, dsc64, dtype)
    else:
        check_f32_tensor("dshift", dshift, dsh64)
        check_f32_tensor("dscale", dscale, dsc64)
    # autograd: the same bits, parameter gradients rounded once
    leaves = [t.clone().requires_grad_() for t in (x, shift, scale)]
    out = F.ln_modulate_ckpt(*leaves, 1e-6, cu, code, group)
    grads = torch.autograd.grad(out, leaves, dy)
    assert same_bits(out.detach(), y) and same_bits(grads[0], dx)
    assert same_bits(grads[1], dshift.to(x.dtype)) and same_bits(grads[2], dscale.to(x.dtype))


@pytest.mark.parametrize("dtype,code", [("bf16", "int8"), ("bf16", "e4m3"), ("f32", "int8"), ("f32", "e4m3")])
@pytest.mark.parametrize("D,group", [(8, 32), (40, 64), (512, 128), (520, 32), (1000, 128), (1536, 64), (2056, 128), (2560, 32),
                                     (3584, 64), (4104, 128), (5120, 128), (6144, 32), (8192, 64)])
def test_ckpt_hidden_sizes(D, group, dtype, code):
    run_ckpt(D, dtype, code, group, B=2, S=37)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,S", [(1, 1), (1, 2), (3, 1), (1, 4099), (4, 777)])
def test_ckpt_rows(B, S, dtype):
    run_ckpt(264, dtype, "int8", 32, B=B, S=S)


@pytest.mark.parametrize("lens", [[1], [0, 5, 0, 0, 1, 300, 0], [3] * 70, [700, 1, 2000, 64, 0], [0] * 40 + [9] + [0] * 40])
@pytest.mark.parametrize("D,dtype,code", [(1536, "bf16", "int8"), (200, "f32", "e4m3")])
def test_ckpt_packed(lens, D, dtype, code):
    run_ckpt(D, dtype, code, 64, lens=lens)


@pytest.mark.parametrize("D,dtype,code,group", [(1536, "bf16", "int8", 128), (5120, "bf16", "e4m3", 32), (200, "f32", "int8", 64),
                                                (8192, "f32", "e4m3", 128), (2568, "bf16", "int8", 64)])
def test_ckpt_per_token(D, dtype, code, group):
    run_ckpt(D, dtype, code, group, B=2, S=131, token=True)


def test_ckpt_large_offsets():
    """Rows whose bytes lie beyond 4 GiB, against the oracle."""
    D, T = 8192, 280000                                                   # x: 4.6 GB
    x = torch.empty(1, T, D, device="cuda", dtype=torch.bfloat16)
    for at in range(0, T, 40000):
        x[0, at:at + 40000].normal_(generator=torch.Generator(device="cuda").manual_seed(at))
    sc = make(3, 1, D, std=0.2)
    y, codes, scales, mean, rstd = lnmod.forward_ckpt(x, sc, sc)
    dx, dsh, dsc = lnmod.backward_ckpt(x, codes, scales, sc, mean, rstd)
    back = lnmod.dequantize(codes, scales, torch.bfloat16)
    sc64, of = to_host64(sc), np.zeros(5, dtype=int)
    for rows in (slice(0, 5), slice(T - 5, T), slice(131070, 131075), slice(262142, 262147)):
        x64 = to_host64(x[0, rows])
        q, s = expect_codes(codes[0, rows], scales[0, rows], x64, "int8", 128)
        assert same_bits(back[0, rows].cpu(), torch.from_numpy(co.decode(q, s, 128)).float().bfloat16())
        y64, mean64, rstd64 = co.ln_forward(x64, sc64, sc64, of, 1e-6)
        check_io_tensor("y", y[0, rows], y64, "bf16")
        check_stats(mean[0, rows], rstd[0, rows], mean64, rstd64)
        check_io_tensor("dx", dx[0, rows], co.ln_backward(x64, co.decode(q, s, 128), sc64, of, mean64, rstd64)[0], "bf16")
    check = x.float().sum((0, 1), dtype=torch.float64)
    assert float((dsh[0].double() - check).abs().max()) <= 1e-5 * float(check.abs().max())


def test_ckpt_rows_with_values_that_are_no_numbers():
    """A row with an infinity or a NaN gives NaN in that row's results alone."""
    x, dy = acts(4, 1, 9, 264), make(5, 1, 9, 264)
    sc = make(6, 1, 264, std=0.2)
    x[0, 3, 100], x[0, 6, 0] = float("inf"), float("nan")
    y, codes, scales, mean, rstd = lnmod.forward_ckpt(x, sc, sc, group=32)
    dx, dsh, dsc = lnmod.backward_ckpt(dy, codes, scales, sc, mean, rstd, group=32)
    bad = torch.tensor([r in (3, 6) for r in range(9)], device="cuda")
    assert dx[0].isnan().all(-1).equal(bad) and not dx[0, ~bad].isnan().any()
    assert dsc.isnan().all() and not dsh.isnan().any()
    fine = torch.zeros_like(x)
    fine[:, ~bad] = x[:, ~bad]
    want = lnmod.forward_ckpt(fine, sc, sc, group=32)
    assert same_bits(y[:, ~bad], want[0][:, ~bad])
    assert same_bits(dx[:, ~bad], lnmod.backward_ckpt(dy, *want[1:3], sc, *want[3:], group=32)[0][:, ~bad])


def test_ckpt_gradients_against_differences():
    """Values that the codes hold exactly (whole numbers up to 127, one of them in each group): the gradients are those of
    the operator itself, and a step along a direction shows it in float64."""
    g = torch.Generator().manual_seed(9)
    T, D, of = 23, 200, np.repeat([0, 1], [15, 8])
    x = torch.randint(-127, 128, (T, D), generator=g).float()
    x[:, ::32] = 127.0
    dy, shift, scale = torch.randn(T, D, generator=g), torch.randn(2, D, generator=g), torch.randn(2, D, generator=g)
    cu = torch.tensor([0, 15, 23], dtype=torch.int32, device="cuda")
    leaves = [t.cuda().requires_grad_() for t in (x, shift, scale)]
    grads = torch.autograd.grad(F.ln_modulate_ckpt(*leaves, 1e-6, cu, "int8", 32), leaves, dy.cuda())
    at = [t.double().numpy() for t in (x, shift, scale)]
    rng = np.random.default_rng(1)
    for k in range(3):
        for _ in range(4):
            d = rng.normal(size=at[k].shape)

            def loss(e):
                moved = [a + e * d if i == k else a for i, a in enumerate(at)]
                return (co.ln_forward(*moved, of, 1e-6)[0] * dy.double().numpy()).sum()

            slope = (loss(1e-5) - loss(-1e-5)) / 2e-5
            # fp32 sums of at most 23 * 200 terms: 1e-5 of the sum of their sizes
            terms = np.abs(to_host64(grads[k]) * d).sum()
            assert abs((to_host64(grads[k]) * d).sum() - slope) <= 1e-5 * terms


# ---- root-mean-square norm with an output in 8 bits ------------------------------------------------------------------------
def check_normed_codes(codes, scales, h64, w64, code, group):
    N, D = h64.shape
    v64, _ = co.rms_forward(h64, w64, 1e-6)
    s, q = co.quotients(v64, code, group)
    gs, got = to_host64(scales).reshape(s.shape), to_host64(codes).reshape(N, D)
    assert (np.abs(gs - s) <= 1.1e-5 * s).all()
    low, high = (co.round_code(np.clip(q * f, -co.LARGEST[code], co.LARGEST[code]), code) for f in (1 - 1e-6, 1 + 1e-6))
    assert ((got >= np.minimum(low, high)) & (got <= np.maximum(low, high))).all()


def run_rms(N, D, dtype, code, group, residual, seed=11):
    print("rms case", N, D, dtype, code, group, residual, flush=True)
    x, w = acts(seed, N, D, dtype=dtype), make(seed + 1, D, dtype=dtype, mean=1.0, std=0.2)
    r = make(seed + 2, N, D, dtype=dtype) if residual else None
    dy, dh = make(seed + 3, N, D, dtype=dtype), make(seed + 4, N, D, dtype=dtype) if residual else None
    codes, scales, h, rstd = lnmod.rmsnorm_quant_forward(x, w, r, 1e-6, code, group)
    assert codes.dtype == KIND[code] and codes.shape == x.shape
    assert scales.shape == ((N, -(-D // group)) if group else (N,))
    if residual:
        assert same_bits(h, (x.float() + r.float()).to(x.dtype))
    else:
        assert h.data_ptr() == x.data_ptr()
    h64, w64 = to_host64(h), to_host64(w)
    _, rstd64 = co.rms_forward(h64, w64, 1e-6)
    assert (np.abs(to_host64(rstd) - rstd64) <= 1e-5 * rstd64).all()
    check_normed_codes(codes, scales, h64, w64, code, group)
    dx, dw = lnmod.rmsnorm_quant_backward(dy, h, w, rstd, dh)
    dx64, dw64 = co.rms_backward(to_host64(dy), h64, w64, rstd64, None if dh is None else to_host64(dh))
    check_io_tensor("dx", dx, dx64, dtype)
    check_f32_tensor("dw", dw, dw64)
    # autograd: what the codes stand for, the same gradients
    leaves = [t.clone().requires_grad_() for t in (x, w) + ((r,) if residual else ())]
    out = F.rms_norm_quant(leaves[0], leaves[1], leaves[2] if residual else None, 1e-6, code, group)
    y = out[1] if residual else out
    assert same_bits(y.detach(), lnmod.dequantize(codes, scales, x.dtype, group))
    grads = torch.autograd.grad(out, leaves, (dh, dy) if residual else dy)
    assert same_bits(grads[0], dx) and same_bits(grads[1], dw.to(x.dtype))
    if residual:
        assert same_bits(out[0].detach(), h) and same_bits(grads[2], dx)


@pytest.mark.parametrize("dtype,code", [("bf16", "e4m3"), ("bf16", "int8"), ("f32", "e4m3"), ("f32", "int8")])
@pytest.mark.parametrize("D,group", [(8, 0), (40, 32), (512, 0), (520, 64), (1000, 0), (1536, 128), (2056, 0), (2560, 64),
                                     (3584, 32), (4104, 128), (5120, 0), (6144, 32), (8192, 0)])
def test_rms_hidden_sizes(D, group, dtype, code):
    run_rms(37, D, dtype, code, group, residual=D % 16 == 0)


@pytest.mark.parametrize("N", [1, 2, 3, 64, 513, 6001])
@pytest.mark.parametrize("group,residual", [(0, True), (128, False)])
def test_rms_rows(N, group, residual):
    run_rms(N, 1536, "bf16", "e4m3", group, residual)


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("D", [264, 5120])
def test_rms_a_scale_for_rows_of_the_smallest_and_largest_products(D, code):
    # h*w of 2^-132 is no normal number: 17 of its bits are left, and three roundings, so s and the quotients are within 1e-5 of
    # the exact ones (and rstd's 1e-5 goes into s); the codes reach the largest one and stay there
    x, w = make(7, 16, D, dtype="f32") * 2.0 ** -50, make(8, D, dtype="f32", mean=1.0, std=0.1) * 2.0 ** -82
    codes, scales, _, _ = lnmod.rmsnorm_quant_forward(x, w, None, 1e-20, code, 0)
    v64, _ = co.rms_forward(to_host64(x), to_host64(w), float(np.float32(1e-20)))
    s, q = co.quotients(v64, code, 0)
    assert (np.abs(to_host64(scales).reshape(s.shape) - s) <= 2.2e-5 * s).all()
    got = to_host64(codes)
    low, high = (co.round_code(np.clip(q * f, -co.LARGEST[code], co.LARGEST[code]), code) for f in (1 - 1e-5, 1 + 1e-5))
    assert ((got >= np.minimum(low, high)) & (got <= np.maximum(low, high))).all()
    # a product beyond float32 counts as an infinity
    codes, scales, _, rstd = lnmod.rmsnorm_quant_forward(make(9, 3, D, dtype="f32") * 2.0 ** 56, w * 2.0 ** 162, None, 1e-6, code, 0)
    assert scales.isnan().all() and not codes.float().any() and bool((rstd > 0).all())


def test_rms_rows_with_values_that_are_no_numbers():
    x, w = acts(4, 6, 264), make(5, 264, mean=1.0, std=0.2)
    r = make(6, 6, 264)
    x[0] = 0
    r[0] = 0
    x[2, 5], r[4, 100] = float("nan"), float("-inf")
    for group in (0, 32):
        codes, scales, h, rstd = lnmod.rmsnorm_quant_forward(x, w, r, code="int8", group=group)
        assert not codes[0].any() and not scales[0].isnan().any()
        s = scales.view(6, -1)
        assert s[2].isnan().all()                                         # rstd is NaN
        # an infinite row: rstd is 0, so its finite values are 0 and the infinite one NaN; a scale for the row covers both
        assert s[4, 0 if group == 0 else 3].isnan()
        assert not s[[0, 1, 3, 5]].isnan().any()
        y = F.rms_norm_quant(x, w, r, code="int8", group=group)[1]
        assert same_bits(y.nan_to_num(7.0), lnmod.dequantize(codes, scales, torch.bfloat16, group).nan_to_num(7.0))
        assert y[2].isnan().all() and y[4].isnan().any() and not y[[0, 1, 3, 5]].isnan().any()


def test_rms_gradients_against_differences():
    g = torch.Generator().manual_seed(10)
    x, r, dy, dh = (torch.randn(11, 200, generator=g) for _ in range(4))
    w = torch.randn(200, generator=g)
    leaves = [t.cuda().requires_grad_() for t in (x, w, r)]
    out = F.rms_norm_quant(*leaves)
    grads = torch.autograd.grad(out, leaves, (dh.cuda(), dy.cuda()))
    at = [(x + r).double().numpy(), w.double().numpy()]                  # h as stored
    rng = np.random.default_rng(2)
    for k in range(2):
        for _ in range(4):
            d = rng.normal(size=at[k].shape)

            def loss(e):
                h, w_ = (a + e * d if i == k else a for i, a in enumerate(at))
                return (co.rms_forward(h, w_, 1e-6)[0] * dy.double().numpy()).sum() + (h * dh.double().numpy()).sum()

            slope = (loss(1e-5) - loss(-1e-5)) / 2e-5
            terms = np.abs(to_host64(grads[k]) * d).sum()
            assert abs((to_host64(grads[k]) * d).sum() - slope) <= 1e-5 * terms


# ---- used together, on streams, in graphs, through the other host path -------------------------------------------------------
def _block(x, r, shift, scale, w, cu):
    """The norms of a block: modulated with a checkpoint, then residual and 8-bit norm; a second checkpoint by hand."""
    y = F.ln_modulate_ckpt(x, shift, scale, 1e-6, cu, "int8", 64)
    h, z = F.rms_norm_quant(y, w, r, code="e4m3", group=128)
    return h, z


def _block_inputs(seed=20, T=300, D=1536):
    x, r = acts(seed, T, D), make(seed + 1, T, D)
    shift, scale, w = make(seed + 2, 3, D, std=0.2), make(seed + 3, 3, D, std=0.2), make(seed + 4, D, mean=1.0, std=0.2)
    cu = torch.tensor([0, 120, 120, T], dtype=torch.int32, device="cuda")
    return x, r, shift, scale, w, cu, make(seed + 5, T, D), make(seed + 6, T, D)


def _block_step(x, r, shift, scale, w, cu, dh, dz):
    leaves = [t.detach().requires_grad_() for t in (x, r, shift, scale, w)]
    h, z = _block(*leaves, cu)
    grads = torch.autograd.grad((h, z), leaves, (dh, dz))
    codes, scales = lnmod.quantize(h.detach(), "e4m3", 32)
    return [h.detach(), z.detach(), *grads, codes, scales, lnmod.dequantize(codes, scales, torch.bfloat16, 32)]


def test_a_run_of_them_together():
    a = _block_inputs()
    x, r, shift, scale, w, cu, dh, dz = a
    got = _block_step(*a)
    # the same chain, each link from the oracle on what the link before it gave
    of = np.repeat([0, 2], [120, 180])
    y, codes, scales, mean, rstd = lnmod.forward_ckpt(x, shift, scale, cu, 1e-6, "int8", 64)
    x64, sc64 = to_host64(x), to_host64(scale)
    y64, mean64, rstd64 = co.ln_forward(x64, to_host64(shift), sc64, of, 1e-6)
    check_io_tensor("y", y, y64, "bf16")
    h = (y.float() + r.float()).bfloat16()
    assert same_bits(got[0], h)
    h64, w64 = to_host64(h), to_host64(w)
    _, r2 = co.rms_forward(h64, w64, 1e-6)
    dyx64, dw64 = co.rms_backward(to_host64(dz), h64, w64, r2, to_host64(dh))
    check_io_tensor("dr", got[3], dyx64, "bf16")
    check_io_tensor("dw", got[6], dw64, "bf16")
    q, s = co.encode(x64, "int8", 64)
    dx64, dsh64, dsc64 = co.ln_backward(to_host64(got[3]), co.decode(q, s, 64), sc64, of, mean64, rstd64)
    check_io_tensor("dx", got[2], dx64, "bf16")
    check_io_tensor("dshift", got[4], dsh64, "bf16")
    check_io_tensor("dscale", got[5], dsc64, "bf16")
    # and twice the same bits
    for u, v in zip(got, _block_step(*a)):
        assert same_bits(u, v)


def test_another_stream():
    a = _block_inputs(30)
    want = _block_step(*a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _block_step(*a)
    side.synchronize()
    for u, v in zip(want, got):
        assert same_bits(u, v)
    x, w = a[0], a[4]
    codes, scales, _, _ = lnmod.rmsnorm_quant_forward(x, w, stream=side)
    back = lnmod.dequantize(codes, scales, torch.float32, 0, stream=side.cuda_stream)
    side.synchronize()
    wc, ws, _, _ = lnmod.rmsnorm_quant_forward(x, w)
    assert same_bits(codes, wc) and same_bits(back, lnmod.dequantize(wc, ws, torch.float32, 0))


def test_two_graphs_with_eager_work_between_their_replays():
    sets = [_block_inputs(40), _block_inputs(50, T=211)]
    graphs, outs = [], []
    side = torch.cuda.Stream()
    for a in sets:
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            _block_step(*a)
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(_block_step(*a))
        graphs.append(g)
    for turn in range(3):
        for k, a in enumerate(sets):
            a[0].copy_(acts(60 + 2 * turn + k, *a[0].shape))
        eager = [_block_step(*a) for a in sets]
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        eager_again = [_block_step(*a) for a in sets]
        torch.cuda.synchronize()
        for k in range(2):
            for u, v, z in zip(eager[k], outs[k], eager_again[k]):
                assert same_bits(u, v) and same_bits(u, z)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("op", ["sample", "token", "packed", "rms", "rms residual"])
def test_the_native_host_path_and_the_python_path_agree(op, dtype):
    """Outputs and gradients bit for bit, also where one of two outputs has no gradient and where saved tensors go through
    hooks."""
    rows, D = ((74, 264) if op == "packed" else (2, 37, 264)), 264
    mod = rows if op == "token" else (4, D) if op == "packed" else (2, D)
    cu = torch.tensor([0, 0, 30, 31, 74], dtype=torch.int32, device="cuda") if op == "packed" else None
    if op.startswith("rms"):
        ts = [make(1, *rows, dtype=dtype), make(2, D, dtype=dtype)] + ([make(3, *rows, dtype=dtype)] if "res" in op else [])
        tail = () if "res" in op else (None,)
        native = lambda *t: F.rms_norm_quant(*t, *tail, 1e-6, "int8", 32)
        python = lambda *t: F._RmsNormQuant.apply(*t, *tail, 1e-6, "int8", 32)
    else:
        ts = [make(1, *rows, dtype=dtype), make(2, *mod, dtype=dtype), make(3, *mod, dtype=dtype)]
        native = lambda *t: F.ln_modulate_ckpt(*t, 1e-6, cu, "e4m3", 64)
        python = lambda *t: F._LnModulateCkpt.apply(*t, cu, 1e-6, "e4m3", 64)
    ts = [t.requires_grad_() for t in ts]

    def results(call, both):
        outs = call(*ts)
        outs = outs if isinstance(outs, tuple) else (outs,)
        used = outs if both else outs[-1:]
        grads = torch.autograd.grad(sum((o.float() * (i + 1.5)).sum() for i, o in enumerate(used)), ts)
        return [o.detach() for o in outs] + list(grads), outs

    for both in (True, False):
        a, outs = results(native, both)
        b, ref = results(python, both)
        assert type(outs[0].grad_fn) is not type(ref[0].grad_fn)
        assert all(same_bits(u, v) for u, v in zip(a, b)) and len(a) == len(b)
    a, b = native(*ts), python(*ts)
    a, b = ((o[0] if isinstance(o, tuple) else o).grad_fn.saved_tensors for o in (a, b))
    assert len(a) == len(b) and all((u is None) == (v is None) and (u is None or same_bits(u, v)) for u, v in zip(a, b))
    with torch.autograd.graph.save_on_cpu():
        assert all(same_bits(u, v) for u, v in zip(results(native, True)[0], results(python, True)[0]))


def test_native_and_python_bindings_agree():
    x, w, r = acts(1, 33, 1432), make(2, 1432), make(3, 33, 1432)
    raw = torch.cuda.current_stream().cuda_stream
    for code, group in (("int8", 32), ("e4m3", 128)):
        a, b = lnmod.quantize(x, code, group), lnmod.quantize(x, code, group, stream=raw)
        assert all(same_bits(u, v) for u, v in zip(a, b))
        assert same_bits(lnmod.dequantize(*a, torch.float32, group), lnmod.dequantize(*a, torch.float32, group, stream=raw))
        for res in (None, r):
            a = lnmod.rmsnorm_quant_forward(x, w, res, 1e-6, code, group)
            b = lnmod.rmsnorm_quant_forward(x, w, res, 1e-6, code, group, stream=raw)
            assert all(same_bits(u, v) for u, v in zip(a, b))
            c = lnmod.rmsnorm_quant_backward(x, a[2], w, a[3], res)
            d = lnmod.rmsnorm_quant_backward(x, a[2], w, a[3], res, stream=raw)
            assert all(same_bits(u, v) for u, v in zip(c, d))
        xs, sc = x.view(3, 11, 1432), make(4, 3, 1432)
        a = lnmod.forward_ckpt(xs, sc, sc, None, 1e-6, code, group)
        b = lnmod.forward_ckpt(xs, sc, sc, None, 1e-6, code, group, stream=raw)
        assert all(same_bits(u, v) for u, v in zip(a, b))
        ws = torch.empty(lnmod.lnmod_backward_ckpt_workspace_bytes(3, 33, 1432), dtype=torch.uint8, device="cuda")
        c = lnmod.backward_ckpt(xs, *a[1:3], sc, *a[3:], group=group)
        d = lnmod.backward_ckpt(xs, *a[1:3], sc, *a[3:], group=group, stream=raw, ws=ws)
        assert all(same_bits(u, v) for u, v in zip(c, d))


def test_refusals_on_the_gpu():
    x, w = make(1, 4, 60, dtype="f32"), make(2, 60, dtype="f32")
    for call in (lambda: lnmod.quantize(x), lambda: lnmod.rmsnorm_quant_forward(x, w), lambda: F.rms_norm_quant(x, w),
                 lambda: lnmod.forward_ckpt(x.view(1, 4, 60), w.view(1, 60), w.view(1, 60))):
        with pytest.raises(lnmod.LnmodError, match="unsupported hidden size"):
            call()
    x = make(1, 4, 65)
    with pytest.raises(ValueError, match="contiguous"):
        lnmod.quantize(x[:, :64])
    flat = make(1, 4 * 64 + 4)[4:].view(4, 64)                            # 8 bytes off
    with pytest.raises(lnmod.LnmodError, match="aligned"):
        lnmod.quantize(flat)
    with pytest.raises(ValueError, match="w is on cpu"):
        lnmod.rmsnorm_quant_forward(make(1, 4, 64), torch.zeros(64, dtype=torch.bfloat16))
