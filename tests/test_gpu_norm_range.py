"""The query and key norm, with the rotation and without, at the ends of float32: a row whose sum of squares is beyond it has
1 / root 0, and zeros for its outputs and its gradient; the rows beside it are what they are without it, bit for bit."""
import pytest
import torch

from paper_2605_17923_amd import functional as F
from paper_2605_17923_amd import lnmod

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])


def zero(t):
    return bool((t == 0).all())


@BOTH
@pytest.mark.parametrize("interleaved", [True, False], ids=["pairs", "halves"])
@pytest.mark.parametrize("per_head", [False, True], ids=["row", "head"])
def test_rows_whose_squares_are_beyond_float32(per_head, interleaved, dtype):
    T, heads, hd, axes = 41, 5, 64, (16, 24, 24)
    g = torch.Generator(device="cuda").manual_seed(3)
    q, dy = (torch.randn(T, heads, hd, generator=g, device="cuda").to(dtype) for _ in range(2))
    w = (torch.rand(hd if per_head else heads * hd, generator=g, device="cuda") + 0.5).to(dtype)
    pos = torch.randint(0, 9, (T, 3), generator=g, device="cuda", dtype=torch.int32)
    table = lnmod.rotary_table(9, axes)
    far = q.clone()
    far[7, 2, 5], far[T - 1, 0, 0], far[12] = 2e19, -torch.finfo(dtype).max, 1.5e19
    outs = []
    for x in (q, far):
        yq, yk, rq, rk = lnmod.qknorm_rotary_forward(x, x, w, w, pos, table, axes, interleaved)
        dq, dk, dwq, dwk = lnmod.qknorm_rotary_backward(dy, dy, x, x, w, w, rq, rk, pos, table, axes, interleaved)
        assert torch.equal(yq, yk) and torch.equal(dq, dk) and torch.equal(dwq, dwk) and bool(dwq.isfinite().all())
        outs.append((yq, dq, rq))
    hit = torch.zeros(T, heads, dtype=torch.bool, device="cuda")
    for row, head in ((7, 2), (T - 1, 0), (12, slice(None))):
        hit[row, head if per_head else slice(None)] = True
    assert zero(outs[1][0][hit]) and zero(outs[1][1][hit]) and zero(outs[1][2][hit if per_head else hit[:, 0]])
    for a, b in zip(outs[0][:2], outs[1][:2]):
        assert torch.equal(a[~hit], b[~hit])


@BOTH
def test_the_norm_without_the_rotation(dtype):
    g = torch.Generator(device="cuda").manual_seed(4)
    q = torch.randn(33, 320, generator=g, device="cuda").to(dtype)
    w = (torch.rand(320, generator=g, device="cuda") + 0.5).to(dtype)
    far = q.clone()
    far[5, 7], far[32] = 2e19, 1.5e19
    x = far.detach().requires_grad_()
    y, z = F.qk_norm(x, q, w, w)
    (dx,) = torch.autograd.grad(y, x, torch.ones_like(y))
    hit = torch.zeros(33, dtype=torch.bool, device="cuda")
    hit[[5, 32]] = True
    assert zero(y[hit]) and zero(dx[hit]) and torch.equal(y[~hit], z[~hit])
