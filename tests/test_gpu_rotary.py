"""Rotary positions with several axes, alone and with the query and key norm, against the formulas in 64 bits.

Bounds.  u = 2^-24 is half a step of float32.  A turned value x c - y s: c and s are rounded (u each), one product and the fused
sum are (u each), so it is off by at most 3 u (|x| + |y|), 4 u with what the products of errors add; then half a step of the
result's type.  1 / root: the squares (u each) are added by at most 64 values of a lane, 6 steps of a wave and 8 waves, all
positive, so their sum is off by 80 u, half of it behind the root, 3 u for product, root and quotient: 44 u < 2^-18.  A normed
value takes two products more.  Backwards, the sum c of a row has the same depth and is off by 2^-17 of the sum of magnitudes.
A sum over n tokens is off by n u of the sum of magnitudes in any order."""
import pytest
import torch

from paper_2605_17923_amd import functional as F
from paper_2605_17923_amd import lnmod

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
EPS = 1e-6


def half_step(t):
    return torch.finfo(t.dtype).eps / 2


def near(got, want, slack, what):
    assert got.shape == want.shape, what
    err = (got.double() - want).abs()
    tol = half_step(got) * want.abs() + slack + 1e-38
    bad = ~(err <= tol)
    assert not bool(bad.any()), "%s: %d values off, worst %.3g of the bound" % (what, int(bad.sum()), float((err / tol).nan_to_num(9e9).max()))


class Case:
    """Inputs on the GPU, and the formulas in 64 bits on the CPU."""

    def __init__(self, dtype=torch.bfloat16, lead=(2, 37), heads=(6, 6), hd=64, axes=(16, 24, 24), interleaved=True, layout="dense",
                 per_head=False, shared=True, rows=61, seed=1):
        g = torch.Generator().manual_seed(seed)
        self.axes, self.interleaved, self.per_head, self.hd, self.lead = axes, interleaved, per_head, hd, lead
        self.table = lnmod.rotary_table(rows, axes)
        ptoks = lead[-1:] if shared else lead
        self.pos = torch.randint(0, rows, ptoks + (len(axes),), generator=g, dtype=torch.int32).cuda()

        def make(n, spare=0):
            if layout == "fused":                      # a part of a wider row
                return (torch.randn(*lead, (n + spare) * hd + 16, generator=g).to(dtype).cuda()[..., 16:16 + n * hd]).unflatten(-1, (n, hd))
            if layout == "heads_first":
                return torch.randn(*lead[:-1], n, lead[-1], hd, generator=g).to(dtype).cuda().transpose(-2, -3)
            return torch.randn(*lead, n, hd, generator=g).to(dtype).cuda()

        self.q, self.k = make(heads[0], 3), make(heads[1], 2)
        self.dq, self.dk = make(heads[0]), make(heads[1])
        width = [hd if per_head else n * hd for n in heads]
        self.wq, self.wk = ((torch.rand(n, generator=g) + 0.5).to(dtype).cuda() for n in width)

    def angles(self):
        of = torch.cat([torch.full((d // 2,), a) for a, d in enumerate(self.axes)])
        freq = torch.cat([10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d) for d in self.axes])
        a = self.pos.cpu().double()[..., of] * freq
        return a.cos().unsqueeze(-2), a.sin().unsqueeze(-2)

    def turn(self, x, back=False, magnitude=False):
        """The rotation; with magnitude |u| + |v| of each pair in both places (0 beyond the turned features)."""
        c, s = self.angles()
        if back:
            s = -s
        R = sum(self.axes)
        a, b = (slice(0, R, 2), slice(1, R, 2)) if self.interleaved else (slice(0, R // 2), slice(R // 2, R))
        y = torch.zeros_like(x) if magnitude else x.clone()
        if magnitude:
            y[..., a] = y[..., b] = x[..., a].abs() + x[..., b].abs()
        else:
            y[..., a] = x[..., a] * c - x[..., b] * s
            y[..., b] = x[..., a] * s + x[..., b] * c
        return y

    def norm(self, x, w):
        x = x.double().cpu()
        w = w.double().cpu().view(-1, self.hd) if not self.per_head else w.double().cpu()
        over = -1 if self.per_head else (-2, -1)
        r = (x.square().mean(over, keepdim=True) + EPS).rsqrt()
        return x, w, r, over

    def check_forward(self, got, x, w, what):
        x, w, r, _ = self.norm(x, w)
        v = x * r * w
        slack = (2.0 ** -18 + 8 * U) * (self.turn(v, magnitude=True) + v.abs())
        near(got.cpu(), self.turn(v), slack, what)

    def check_backward(self, dx, dw, x, w, dy, what):
        dw_t = dw.cpu()
        x, w, r, over = self.norm(x, w)
        dy = dy.double().cpu()
        g, gm = self.turn(dy, back=True), self.turn(dy, magnitude=True) + dy.abs()
        xhat = x * r
        c = (g * w * xhat).mean(over, keepdim=True)
        slack = 2.0 ** -17 * r * (gm * w.abs() + xhat.abs() * (gm * w.abs() * xhat.abs()).mean(over, keepdim=True))
        near(dx.cpu(), r * (g * w - xhat * c), slack, what + " dx")
        dims = tuple(range(x.dim() - (1 if self.per_head else 2)))
        n = x[..., 0].numel() if self.per_head else x[..., 0, 0].numel()
        near(dw_t, (g * xhat).sum(dims).reshape(-1), (2.0 ** -17 + n * U) * (gm * xhat.abs()).sum(dims).reshape(-1), what + " dw")


SHAPES = [dict(),
          dict(lead=(1, 1), heads=(40, 40), hd=128, axes=(44, 42, 42)),
          dict(lead=(3, 29), heads=(12, 4), hd=128, axes=(32, 48, 48), interleaved=False),
          dict(lead=(71,), heads=(5, 1), hd=72, axes=(24, 24, 24), layout="fused"),
          dict(lead=(2, 19), heads=(1, 1), hd=8, axes=(2, 2, 4)),
          dict(lead=(2, 19), heads=(3, 7), hd=8, axes=(8,), interleaved=False),
          dict(lead=(2, 33), heads=(24, 8), hd=96, axes=(32, 16, 16), interleaved=False, layout="heads_first"),
          dict(lead=(2, 18), heads=(9, 9), hd=64, axes=(6, 10), layout="heads_first"),
          dict(lead=(130,), heads=(32, 2), hd=256, axes=(64, 96, 96)),
          dict(lead=(2, 40), heads=(31, 17), hd=136, axes=(8, 8, 8, 8), shared=False),
          dict(lead=(515,), heads=(64, 64), hd=128, axes=(64, 64), interleaved=False, layout="fused"),
          dict(lead=(2, 1025), heads=(2, 3), hd=40, axes=(10, 10, 20), layout="fused")]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_rotation_and_its_gradient(shape, dtype):
    c = Case(dtype, **SHAPES[shape])
    q, k = c.q.detach().requires_grad_(), c.k.detach().requires_grad_()
    ys = F.rotary(q, k, c.pos, c.table, c.axes, c.interleaved)
    grads = torch.autograd.grad(ys, (q, k), (c.dq, c.dk))
    for y, x, d, dy, name in zip(ys, (c.q, c.k), grads, (c.dq, c.dk), "qk"):
        assert y.is_contiguous() and d.is_contiguous()
        x, dy = x.double().cpu(), dy.double().cpu()
        near(y.detach().cpu(), c.turn(x), 4 * U * c.turn(x, magnitude=True), name)
        near(d.cpu(), c.turn(dy, back=True), 4 * U * c.turn(dy, magnitude=True), "d" + name)
    R = sum(c.axes)
    assert torch.equal(ys[0][..., R:].detach(), c.q[..., R:])                     # beyond the turned features
    alone = F.rotary(c.q, None, c.pos, c.table, c.axes, c.interleaved)
    assert torch.equal(alone, ys[0])
    direct = lnmod.rotary(c.q, c.k, c.pos, c.table, c.axes, c.interleaved)
    assert torch.equal(direct[0], ys[0]) and torch.equal(direct[1], ys[1])


@pytest.mark.parametrize("per_head", [False, True], ids=["row", "head"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_norm_with_rotation_and_its_gradients(shape, dtype, per_head):
    c = Case(dtype, per_head=per_head, **SHAPES[shape])
    leaves = tuple(t.detach().requires_grad_() for t in (c.q, c.k, c.wq, c.wk))
    ys = F.qk_norm_rotary(*leaves, c.pos, c.table, c.axes, c.interleaved, EPS)
    dq, dk, dwq, dwk = torch.autograd.grad(ys, leaves, (c.dq, c.dk))
    c.check_forward(ys[0].detach(), c.q, c.wq, "q")
    c.check_forward(ys[1].detach(), c.k, c.wk, "k")
    c.check_backward(dq, dwq, c.q, c.wq, c.dq, "q")
    c.check_backward(dk, dwk, c.k, c.wk, c.dk, "k")
    qo, ko, rq, rk = lnmod.qknorm_rotary_forward(c.q, c.k, c.wq, c.wk, c.pos, c.table, c.axes, c.interleaved, EPS)
    assert torch.equal(qo, ys[0]) and torch.equal(ko, ys[1])
    args = (c.dq, c.dk, c.q, c.k, c.wq, c.wk, rq, rk, c.pos, c.table, c.axes, c.interleaved)
    a = lnmod.qknorm_rotary_backward(*args)
    assert a[2].dtype == torch.float32 and torch.equal(a[0], dq) and torch.equal(a[2].to(dtype), dwq) and torch.equal(a[3].to(dtype), dwk)
    for x, y in zip(a, lnmod.qknorm_rotary_backward(*args)):
        assert torch.equal(x, y)                                                  # the same bits again
