"""The 8-bit operators at the edges of what their calls allow: values next to the largest float, gradients that share a
consumer, transforms, threads, another stream.  Compared bit for bit unless said otherwise."""
import threading

import pytest
import torch

from paper_2605_17923_amd import functional as F
from paper_2605_17923_amd import lnmod

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def make(seed, *shape, dtype="bf16", mean=0.0, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std + mean).to(DT[dtype]).cuda()


def bits(t):
    return t.contiguous().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


def same_bits(a, b):
    return a.dtype == b.dtype and a.shape == b.shape and torch.equal(bits(a), bits(b))


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_finite_groups_stay_finite(dtype, code):
    """Masks of the type's lowest value, and the floats next to the largest one, come back finite: the float32 product of
    code and scale, held to the largest float."""
    top = torch.finfo(DT[dtype]).max
    x = make(3, 40, 96, dtype=dtype)
    x[0, 5:] = -top
    x[1] = top
    x[2, 32], x[3, 95] = top, -top
    steps = torch.tensor([top], dtype=DT[dtype]).view(torch.int16 if dtype == "bf16" else torch.int32).item()
    for k in range(32):                                                    # the k-th below the largest
        x[4 + k, ::7] = torch.tensor([steps - k]).to(torch.int16 if dtype == "bf16" else torch.int32).view(DT[dtype]).item()
    x[36, 0] = float("inf")
    codes, scales = lnmod.quantize(x, code, 32)
    back = lnmod.dequantize(codes, scales, x.dtype, 32)
    s = scales.cpu().double().repeat_interleave(32, 1)
    want = (codes.cpu().double() * s).float()                              # one rounding; infinite beyond the largest float
    big = torch.finfo(torch.float32).max
    want = torch.where(s.isfinite(), want.clamp(-big, big), want).to(x.dtype)
    assert same_bits(back.cpu().nan_to_num(7.0), want.nan_to_num(7.0)) and torch.equal(back.cpu().isnan(), want.isnan())
    assert torch.equal(back.isfinite(), scales.isfinite().repeat_interleave(32, 1))
    assert back[1].eq(top).all() and back[0, 5:].eq(-top).all()
    # scales of the caller's own: code*s as it is
    scales[0], scales[1], scales[2, 0] = float("inf"), float("-inf"), float("nan")
    back = lnmod.dequantize(codes, scales, x.dtype, 32)
    want = (codes.cpu().double() * scales.cpu().double().repeat_interleave(32, 1)).to(x.dtype)[:3]
    same = same_bits(back[:2].cpu().nan_to_num(7.0, 8.0, 9.0), want[:2].nan_to_num(7.0, 8.0, 9.0))
    assert same and back[2, :32].isnan().all()


def test_finite_normed_rows_stay_finite():
    big = torch.finfo(torch.float32).max
    x = torch.ones(5, 64, device="cuda")
    w = torch.full((64,), big, device="cuda")
    w[40:] = -1.0
    for code in ("int8", "e4m3"):
        codes, scales, _, rstd = lnmod.rmsnorm_quant_forward(x, w, None, 1e-30, code, 32)
        assert rstd.eq(1.0).all() and scales.isfinite().all()
        y = F.rms_norm_quant(x, w, None, 1e-30, code, 32)
        assert y.isfinite().all() and y[:, :32].eq(big).all()
        assert same_bits(y, lnmod.dequantize(codes, scales, torch.float32, 32))


@pytest.mark.parametrize("path", ["native", "python"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_gradients_of_x_and_of_the_residual_share_no_memory(dtype, path):
    """With views in front of the operator the leaves' .grad are made of the very tensors that the backward returns."""
    N, D = 37, 264
    call = F.rms_norm_quant if path == "native" else (lambda *t: F._RmsNormQuant.apply(*t, 1e-6, "e4m3", 0))
    a, b, w = (make(k, *s, dtype=dtype).requires_grad_() for k, s in ((1, (N * D,)), (2, (N * D,)), (3, (D,))))
    total = 0.0
    for turn in range(3):
        dh, dy = make(10 + turn, N, D, dtype=dtype), make(20 + turn, N, D, dtype=dtype)
        torch.autograd.backward(call(a.view(N, D), w, b.view(N, D)), (dh, dy))
        h, rstd = lnmod.rmsnorm_quant_forward(a.detach().view(N, D), w.detach(), b.detach().view(N, D))[2:]
        dx = lnmod.rmsnorm_quant_backward(dy, h, w.detach(), rstd, dh)[0].view(-1)
        total = dx if turn == 0 else total + dx
        for leaf in (a, b):
            assert same_bits(leaf.grad, total), turn
    a.grad.zero_()
    assert same_bits(b.grad, total)
    x, r = (t.detach().view(N, D).requires_grad_() for t in (a, b))
    gx, gr = torch.autograd.grad(call(x, w, r), (x, r), (dh, dy))
    assert same_bits(gx, gr) and gx.untyped_storage().data_ptr() != gr.untyped_storage().data_ptr()
    # one of the two alone, and one tensor in both places
    for one in (x, r):
        assert same_bits(torch.autograd.grad(call(x, w, r), one, (dh, dy))[0], gx)
        frozen = [t if t is one else t.detach() for t in (x, r)]
        assert same_bits(torch.autograd.grad(call(frozen[0], w, frozen[1]), one, (dh, dy))[0], gx)
    both, = torch.autograd.grad(call(x, w, x), x, (dh, dy))
    h, rstd = lnmod.rmsnorm_quant_forward(x.detach(), w.detach(), x.detach())[2:]
    assert same_bits(both, lnmod.rmsnorm_quant_backward(dy, h, w.detach(), rstd, dh)[0] * 2)


@pytest.mark.parametrize("N,D", [(1, 8), (257, 1536), (4099, 2600), (9001, 5120)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_second_copy_is_the_first(N, D, dtype):
    dy, h, w, dh = (make(k, *s, dtype=dtype) for k, s in ((1, (N, D)), (2, (N, D)), (3, (D,)), (4, (N, D))))
    rstd = lnmod.rmsnorm_quant_forward(h, w)[3]
    for along in (dh, None):
        dx, dw = lnmod.rmsnorm_quant_backward(dy, h, w, rstd, along)
        got = lnmod._rmsnorm_quant_backward(dy, h, w, rstd, along, own_dr=True)
        assert all(same_bits(u, v) for u, v in zip(got, (dx, dw, dx)))


def test_transforms_are_refused():
    x, sh, sc = (make(k, 3, *s, dtype="f32") for k, s in ((1, (2, 8, 64)), (2, (2, 64)), (3, (2, 64))))
    r, w = make(4, 3, 2, 8, 64, dtype="f32"), make(5, 64, dtype="f32")
    ln = lambda t: F.ln_modulate_ckpt(t, sh[0], sc[0], group=32)
    rms = lambda t: F.rms_norm_quant(t, w, r[0])[1]
    with pytest.raises(RuntimeError):
        torch.func.vmap(F.ln_modulate_ckpt)(x, sh, sc)
    with pytest.raises(RuntimeError):
        torch.func.vmap(lambda t, u: F.rms_norm_quant(t, w, u)[1])(x, r)
    with pytest.raises(RuntimeError):
        torch.func.vmap(lambda t: lnmod.quantize(t)[0])(x)
    for call in (ln, rms):
        with pytest.raises(RuntimeError):
            torch.func.grad(lambda t: call(t).sum())(x[0])
        with torch.autograd.forward_ad.dual_level(), pytest.raises(RuntimeError):
            call(torch.autograd.forward_ad.make_dual(x[0], x[0]))
        leaf = x[0].clone().requires_grad_()
        g = torch.randn_like(leaf).requires_grad_()
        first, = torch.autograd.grad(call(leaf), leaf, g, create_graph=True)
        assert not first.requires_grad                                     # no half-connected second derivative


def test_calls_from_several_threads():
    """Each thread on a stream of its own, all at once, forwards and backwards: what one thread alone gives."""
    D, N, turns = 1536, 700, 8
    sets = [(make(k, N, D), make(k + 10, N, D), make(k + 20, 2, D, std=0.2), make(k + 30, D, mean=1.0, std=0.2), make(k + 40, N, D))
            for k in range(4)]
    cu = torch.tensor([0, 300, N], dtype=torch.int32, device="cuda")

    def step(x, r, mod, w, dy):
        x, r, mod, w = (t.detach().requires_grad_() for t in (x, r, mod, w))
        y = F.ln_modulate_ckpt(x, mod, mod, 1e-6, cu, "e4m3", 64)
        h, z = F.rms_norm_quant(y, w, r, code="int8", group=128)
        grads = torch.autograd.grad((h, z), (x, r, mod, w), (dy, dy))
        codes, scales = lnmod.quantize(z.detach(), "int8", 32)
        return [h.detach(), z.detach(), *grads, codes, scales, lnmod.dequantize(codes, scales, torch.bfloat16, 32)]

    want = [step(*s) for s in sets]
    torch.cuda.synchronize()
    got, errors = [None] * 4, []

    def work(k):
        try:
            torch.cuda.set_device(0)
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                got[k] = [step(*sets[k]) for _ in range(turns)]
            stream.synchronize()
        except BaseException as e:                                         # noqa: BLE001  (shown by the assertion below)
            errors.append(e)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    assert not errors and not any(t.is_alive() for t in threads)
    for k in range(4):
        for outs in got[k]:
            assert all(same_bits(u, v) for u, v in zip(outs, want[k]))


@pytest.mark.parametrize("op", ["sample", "packed", "rms"])
def test_a_gradient_that_nobody_asks_for(op):
    """One output of the norm used, or one leaf frozen: the others' gradients keep their bits."""
    D = 264
    cu = torch.tensor([0, 5, 5, 74], dtype=torch.int32, device="cuda") if op == "packed" else None
    if op == "rms":
        ts = [make(1, 74, D), make(2, D), make(3, 74, D)]
        call = lambda *t: F.rms_norm_quant(*t, 1e-6, "int8", 32)[1]
    else:
        ts = [make(1, *((74, D) if cu is not None else (1, 74, D))), make(2, 1 if cu is None else 3, D), make(3, 1 if cu is None else 3, D)]
        call = lambda *t: F.ln_modulate_ckpt(*t, 1e-6, cu, "int8", 32)
    dy = make(4, *ts[0].shape)
    leaves = [t.requires_grad_() for t in ts]
    want = torch.autograd.grad(call(*leaves), leaves, dy)
    for k in range(3):
        some = [t if i == k else t.detach() for i, t in enumerate(leaves)]
        got, = torch.autograd.grad(call(*some), leaves[k], dy)
        assert same_bits(got, want[k]), k


def test_a_mean_of_squares_beyond_float32():
    """rstd is formed in float32, as the header says: 0 where the mean of squares is beyond it."""
    x, w = make(1, 3, 64, dtype="f32"), make(2, 64, dtype="f32")
    x[1] = 1e25
    for group in (0, 32):
        codes, scales, _, rstd = lnmod.rmsnorm_quant_forward(x, w, None, 1e-6, "int8", group)
        assert rstd[1] == 0 and (rstd[[0, 2]] > 0).all() and not codes[1].any() and codes[[0, 2]].any(-1).all()
        assert scales.isfinite().all()


def test_offsets_beyond_four_gib():
    """quantize, the norm and its backward (both forms) on rows whose bytes lie beyond 4 GiB: what the same rows give alone."""
    D, N = 8192, 280000                                                    # 4.6 GB each
    x, r = (torch.empty(N, D, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    for k, t in enumerate((x, r)):
        for at in range(0, N, 40000):
            t[at:at + 40000].normal_(generator=torch.Generator(device="cuda").manual_seed(at + k))
    w = make(3, D, mean=1.0, std=0.2)
    parts = [slice(a, a + 5) for a in (0, 131070, 262142, N - 5)]
    codes, scales = lnmod.quantize(x, "int8", 128)
    for p in parts:
        want = lnmod.quantize(x[p].contiguous(), "int8", 128)
        assert same_bits(codes[p], want[0]) and same_bits(scales[p], want[1]), p
    del codes, scales
    codes, scales, h, rstd = lnmod.rmsnorm_quant_forward(x, w, r, 1e-6, "e4m3", 128)
    alone = [lnmod.rmsnorm_quant_forward(x[p].contiguous(), w, r[p].contiguous(), 1e-6, "e4m3", 128) for p in parts]
    for p, want in zip(parts, alone):
        assert same_bits(h[p], want[2])
        # sums of squares in another order where the launch shape differs: codes and scales as far as rstd is the same
        rows = rstd[p] == want[3]
        assert rows.any() and bool(((rstd[p] - want[3]).abs() <= 1e-6 * want[3]).all())
        assert same_bits(codes[p][rows].float(), want[0][rows].float()) and same_bits(scales[p][rows], want[1][rows])
    del codes, scales
    dx, _, dr = lnmod._rmsnorm_quant_backward(x, h, w, rstd, r, own_dr=True)
    assert same_bits(dx, dr)
    for p in parts:
        g, hhat = x[p].double() * w.double(), h[p].double() * rstd[p].double()[:, None]
        ref = r[p].double() + rstd[p].double()[:, None] * (g - hhat * (g * hhat).mean(-1, keepdim=True))
        # one rounding to bf16, 2^-8 of the value at most, and fp32 sums
        assert bool(((dx[p].double() - ref).abs() <= ref.abs() * 2.0 ** -8 + 1e-5 * ref.abs().max()).all())
    torch.cuda.empty_cache()
