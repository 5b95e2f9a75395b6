"""The 8-bit row operators at every entry of their launch-shape tables: each width class of 512 features, each class of sizes,
both element types, one sample, several segments and a modulation row per token.  The reference is plain torch in float64 on the
device (the small tests compare with the CPU oracle); bounds as in parity_util: bf16 results within one unit of the
last place of the rounded reference plus 1e-5 of the largest, float32 results and sums within 1e-5 of the largest."""
import pytest
import torch

from paper_2605_17923_amd import lnmod

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(autouse=True)
def _memory():
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def rows_of(mb, D, dtype):
    return max(1, int(mb * 1e6 / (D * (2 if dtype == "bf16" else 4))))


def close(name, got, ref):
    assert got.shape == ref.shape
    if ref.numel() == 0:
        return
    assert bool(torch.isfinite(got).all()), name
    err = (got.double() - ref).abs()
    top = float(ref.abs().max())
    if got.dtype == torch.bfloat16:
        rounded = ref.to(torch.bfloat16).double()
        _, expo = torch.frexp(rounded.abs().clamp_min(2.0 ** -126))
        bound = torch.ldexp(torch.full_like(rounded, 1.0001), expo - 8) + 1e-5 * top
        err = (got.double() - rounded).abs()
    else:
        bound = torch.full_like(err, 1e-5 * top + 1e-30)
    assert not bool((err > bound).any()), "%s: %d beyond, worst %.3e of %.3e" % (name, int((err > bound).sum()), float(err.max()), top)


def inputs(seed, *shapes, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(s, generator=g, device="cuda").to(DT[dtype]) for s in shapes]


def decoded(codes, scales, group):
    D = codes.shape[-1]
    wide = scales.double().repeat_interleave(group, -1)[..., :D]
    return codes.double() * wide


def run_ckpt(D, T, dtype, code, group, cuts=None, token=False):
    print("ckpt", D, T, dtype, code, group, "token" if token else cuts, flush=True)
    n = 1 if cuts is None else len(cuts) - 1
    shape = (T, D) if cuts is not None else (1, T, D)
    mod = shape if token else (n, D)
    x, dy, shift, scale = inputs(D + T, shape, shape, mod, mod, dtype=dtype)
    cu = None if cuts is None else torch.tensor(cuts, dtype=torch.int32, device="cuda")
    y, codes, scales, mean, rstd = lnmod.forward_ckpt(x, shift, scale, cu, 1e-6, code, group)
    qc, qs = lnmod.quantize(x, code, group)
    assert torch.equal(codes.view(torch.uint8), qc.view(torch.uint8)) and torch.equal(scales, qs)
    dx, dsh, dsc = lnmod.backward_ckpt(dy, codes, scales, scale, mean, rstd, cu, group)
    again = lnmod.backward_ckpt(dy, codes, scales, scale, mean, rstd, cu, group)
    assert all(torch.equal(a, b) for a, b in zip((dx, dsh, dsc), again))
    if token:
        assert torch.equal(dsh, dy)
    flat = lambda t: t.reshape(-1, D)
    ends = [0, T] if cuts is None else cuts
    for m in range(n):
        r = slice(ends[m], ends[m + 1])
        v, d = flat(x)[r].double(), flat(dy)[r].double()
        sc, sh = (flat(t)[r].double() if token else t[m].double() for t in (scale, shift))
        mu = v.mean(-1, keepdim=True)
        rs = ((v - mu).square().mean(-1, keepdim=True) + 1e-6).rsqrt()
        close("y", flat(y)[r], (v - mu) * rs * (1 + sc) + sh)
        del v
        xhat = (decoded(flat(codes)[r], flat_scales(scales)[r], group) - mu) * rs
        g = d * (1 + sc)
        close("dx", flat(dx)[r], rs * (g - g.mean(-1, keepdim=True) - xhat * (g * xhat).mean(-1, keepdim=True)))
        del g
        if token:
            close("dscale", flat(dsc)[r], d * xhat)
        else:
            close("dshift", dsh[m], d.sum(0))
            close("dscale", dsc[m], (d * xhat).sum(0))


def flat_scales(s):
    return s.reshape(-1, s.shape[-1])


# a width in each class, on and off whole lines, and one size on each side of every line between the tables
@pytest.mark.parametrize("mb", [8, 14, 48, 70, 220])
@pytest.mark.parametrize("col", range(1, 17))
def test_checkpoint_tables_bf16(col, mb):
    D = 512 * col - (64, 8, 256)[(col + mb) % 3]
    run_ckpt(D, rows_of(mb, D, "bf16"), "bf16", ("int8", "e4m3")[(col + mb // 2) % 2], (32, 64, 128)[col % 3])


@pytest.mark.parametrize("mb", [8, 14, 60])
@pytest.mark.parametrize("col", range(1, 17))
def test_checkpoint_tables_f32(col, mb):
    D = 512 * col - (64, 8, 256)[(col + mb) % 3]
    run_ckpt(D, rows_of(mb, D, "f32"), "f32", ("int8", "e4m3")[col % 2], (32, 64, 128)[col % 3])


@pytest.mark.parametrize("mb", [14, 70])
@pytest.mark.parametrize("col", range(1, 17))
def test_checkpoint_tables_several_segments(col, mb):
    D = 512 * col - (64, 8, 256)[col % 3]
    T = rows_of(mb, D, "bf16")
    cuts = [0, 0, 1, T // 7, T // 7 + 3, T // 2, T // 2, T - 5, T]
    run_ckpt(D, T, "bf16", "int8", 128, cuts=cuts)


@pytest.mark.parametrize("mb", [8, 14, 210])
@pytest.mark.parametrize("col", range(1, 17))
def test_checkpoint_tables_per_token(col, mb):
    D = 512 * col - (64, 8, 256)[(col + mb) % 3]
    dtype = "f32" if (col + mb) % 4 == 3 else "bf16"
    run_ckpt(D, rows_of(mb, D, dtype), dtype, "int8", (32, 64, 128)[col % 3], token=True)


def run_rms(D, N, dtype, code, group, residual):
    print("rms", D, N, dtype, code, group, residual, flush=True)
    x, r, dy, dh, w = inputs(D + N, (N, D), (N, D), (N, D), (N, D), (D,), dtype=dtype)
    r, dh = (r, dh) if residual else (None, None)
    codes, scales, h, rstd = lnmod.rmsnorm_quant_forward(x, w, r, 1e-6, code, group)
    if residual:
        assert torch.equal(h, (x.float() + r.float()).to(x.dtype))
    h64, w64 = h.double(), w.double()
    rs = (h64.square().mean(-1, keepdim=True) + 1e-6).rsqrt()
    close("rstd", rstd.view(-1, 1), rs)
    hhat = h64 * rs
    v = hhat * w64
    # the exact quotient, off by 4e-7 at most, decides the code: within half a step of it, 2^-4 of an e4m3 value
    wide = (scales.view(N, 1) if group == 0 else scales.repeat_interleave(group, -1)[:, :D]).double()
    if group == 0:
        close("scales", scales, v.abs().amax(-1) / (127 if code == "int8" else 448))
    q = v / wide
    off = (codes.double() - q).abs()
    half = 0.5 if code == "int8" else torch.maximum(q.abs() * 2.0 ** -4, torch.full_like(q, 2.0 ** -10))
    assert bool((off <= half + q.abs() * 1e-6 + 1e-9).all())
    assert float(codes.double().abs().max()) == (127 if code == "int8" else 448)
    y = lnmod._rmsnorm_quant(x, w, r, 1e-6, code, group, values=True)[2]
    assert torch.equal(y, lnmod.dequantize(codes, scales, x.dtype, group))
    del v, q, off, wide
    dx, dw = lnmod.rmsnorm_quant_backward(dy, h, w, rstd, dh)
    g = dy.double() * w64
    ref = rs * (g - hhat * (g * hhat).mean(-1, keepdim=True))
    close("dx", dx, ref if dh is None else ref + dh.double())
    close("dw", dw, (dy.double() * hhat).sum(0))


@pytest.mark.parametrize("mb", [8, 30, 70, 220])
@pytest.mark.parametrize("col", range(1, 17))
def test_rms_tables_bf16(col, mb):
    D = 512 * col - (64, 8, 256)[(col + mb) % 3]
    run_rms(D, rows_of(mb, D, "bf16"), "bf16", ("e4m3", "int8")[(col + mb // 2) % 2], (0, 32, 64, 128)[(col + mb // 2) % 4],
            (col + mb // 10) % 3 != 0)


@pytest.mark.parametrize("mb", [8, 30, 70])
@pytest.mark.parametrize("col", range(1, 17))
def test_rms_tables_f32(col, mb):
    D = 512 * col - (64, 8, 256)[(col + mb) % 3]
    run_rms(D, rows_of(mb, D, "f32"), "f32", ("e4m3", "int8")[col % 2], (0, 32, 64, 128)[(col + mb // 2) % 4], col % 2 == 0)


@pytest.mark.parametrize("mb,D,group", [(10, 1536, 128), (40, 5120, 32), (350, 2048, 64), (20, 2600, 128), (330, 1000, 64)])
@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_quantize_sizes(mb, D, group, code):
    N = rows_of(mb, D, "bf16")
    print("quantize", N, D, group, code, flush=True)
    x, = inputs(mb, (N, D), dtype="bf16")
    codes, scales = lnmod.quantize(x, code, group)
    pad = torch.nn.functional.pad(x.double(), (0, -D % group)).unflatten(-1, (-1, group))
    s = (pad.abs().amax(-1) / (127.0 if code == "int8" else 448.0)).float()
    assert torch.equal(scales, s)
    p = pad * (1.0 / s.double()).float().double().unsqueeze(-1)
    p = (p.round() if code == "int8" else p.float().to(torch.float8_e4m3fn).double()).flatten(-2)[:, :D]
    assert torch.equal(codes.double(), p)
    assert torch.equal(lnmod.dequantize(codes, scales, torch.bfloat16, group), decoded(codes, scales, group).float().bfloat16())


def test_two_streams_at_once():
    """Calls that overlap on two streams, each with memory of its own, give what they give one after the other."""
    D, T = 2056, 9001
    sets = []
    for k in range(2):
        x, r, dy, dh = inputs(k, (1, T, D), (1, T, D), (1, T, D), (1, T, D), dtype="bf16")
        sc, w = inputs(9 + k, (1, D), (D,), dtype="bf16")
        sets.append((x, r, dy, dh, sc, w))

    def step(x, r, dy, dh, sc, w):
        y, codes, scales, mean, rstd = lnmod.forward_ckpt(x, sc, sc, None, 1e-6, "e4m3", 64)
        c, s, h, rs = lnmod.rmsnorm_quant_forward(y, w, r)
        d = lnmod.rmsnorm_quant_backward(dy, h, w, rs, dh)
        return (y, codes, scales, c, s, h) + d + lnmod.backward_ckpt(d[0], codes, scales, sc, mean, rstd, None, 64)

    want = [step(*a) for a in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[], []]
    for _ in range(6):
        for k, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[k].append(step(*sets[k]))
    torch.cuda.synchronize()
    for k in range(2):
        for out in got[k]:
            for a, b in zip(out, want[k]):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


# rows that end inside a group: several to a wave, or lengthened; the codes and scales are those of the rows with zeros behind
# them, and codes of such rows stand for the same values.  Sizes of each launch rule (1, 2 and 4 pieces a wave).
@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,N,D,group", [("bf16", 70001, 8, 32), ("bf16", 4001, 24, 128), ("bf16", 300, 40, 32), ("bf16", 9000, 72, 64),
                                             ("bf16", 130003, 72, 128), ("bf16", 50001, 200, 32), ("bf16", 20011, 504, 128),
                                             ("bf16", 9001, 1000, 64), ("bf16", 800017, 200, 128), ("bf16", 33001, 5000, 128),
                                             ("f32", 70001, 8, 64), ("f32", 50001, 200, 128), ("f32", 7001, 520, 32),
                                             ("f32", 1025, 1432, 128), ("bf16", 3, 1 << 20, 128), ("bf16", 5, (1 << 20) - 8, 128)])
def test_quantize_rows_that_end_inside_a_group(dtype, N, D, group, code):
    g = torch.Generator(device="cuda").manual_seed(D + N)
    x = (torch.randn(N, D, generator=g, device="cuda") * torch.rand(N, 1, generator=g, device="cuda") * 8).to(DT[dtype])
    wide = -(-D // group) * group
    padded = torch.zeros(N, wide, dtype=DT[dtype], device="cuda")
    padded[:, :D] = x
    codes, scales = lnmod.quantize(x, code, group)
    want, wscales = lnmod.quantize(padded, code, group)
    assert torch.equal(scales, wscales)
    assert torch.equal(codes.view(torch.uint8), want.view(torch.uint8)[:, :D].contiguous())
    assert torch.equal(lnmod.dequantize(codes, scales, DT[dtype], group),
                       lnmod.dequantize(want, wscales, DT[dtype], group)[:, :D].contiguous())
    # one scale for a row: the same values from groups that share it
    row = torch.rand(N, generator=g, device="cuda") + 0.5
    shared = row[:, None].expand(N, wscales.shape[1]).contiguous()
    assert torch.equal(lnmod.dequantize(codes, row, DT[dtype], 0),
                       lnmod.dequantize(want, shared, DT[dtype], group)[:, :D].contiguous())


# Backwards where the waves of a block hold rows of their own and add what they have summed: from one row to more than a
# step of the whole grid, last steps that some waves have no row in, segments shorter than a block's rows.
@pytest.mark.parametrize("rows", [1, 2, 255, 257, 600, 1025, 3100, 12289])
@pytest.mark.parametrize("D,dtype", [(200, "bf16"), (1000, "bf16"), (1536, "bf16"), (2000, "bf16"), (2560, "bf16"), (400, "f32"),
                                     (1024, "f32")])
def test_rows_of_one_wave(D, dtype, rows):
    run_ckpt(D, rows, dtype, "int8", 64)
    run_ckpt(D, rows + 40, dtype, "e4m3", 128, cuts=[0, 0, 1, 2, rows // 2 + 2, rows + 2, rows + 2, rows + 39, rows + 40])
    run_rms(D, rows, dtype, "e4m3", 64, True)
    run_rms(D, rows, dtype, "int8", 0, False)


@pytest.mark.parametrize("D", [200, 1000, 1496, 2504])
def test_rows_of_one_wave_in_the_long_launches(D):
    for residual in (True, False):
        run_rms(D, rows_of(60, D, "bf16"), "bf16", "e4m3", 128, residual)
        run_rms(D, rows_of(60, D, "f32"), "f32", "e4m3", 128, residual)
    run_ckpt(D, rows_of(60, D, "f32"), "f32", "int8", 128, cuts=[0, 700, 700, 701, 3000, rows_of(60, D, "f32")])
