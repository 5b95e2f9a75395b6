"""The rotation and the query and key norm with it: positions without an angle, values that are no numbers, gaps between heads,
offsets beyond 32 bits, second derivatives, both host paths, streams, graphs, threads, and a run of the operators together."""
import threading

import pytest
import torch

from paper_2605_17923_amd import functional as F
from paper_2605_17923_amd import lnmod
from test_gpu_rotary import EPS, U, Case, half_step, near

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
PAIRS = pytest.mark.parametrize("interleaved", [True, False], ids=["pairs", "halves"])
bf = torch.bfloat16


def same(a, b):
    """The same bits, NaN where NaN is."""
    return a.shape == b.shape and a.dtype == b.dtype and bool(((a == b) | (a.isnan() & b.isnan())).all())


def axis_features(axes, interleaved, axis):
    """The features of an axis' pairs."""
    first = sum(axes[:axis]) // 2
    pairs = torch.arange(first, first + axes[axis] // 2)
    return torch.cat([2 * pairs, 2 * pairs + 1]) if interleaved else torch.cat([pairs, pairs + sum(axes) // 2])


@BOTH
@PAIRS
@pytest.mark.parametrize("bad", [-1, 61, 2 ** 31 - 1, -2 ** 31])
def test_a_position_outside_the_table_makes_its_axis_nan(bad, interleaved, dtype):
    c = Case(dtype, lead=(2, 37), heads=(6, 2), hd=72, axes=(16, 24, 16), interleaved=interleaved, shared=False)
    want = lnmod.rotary(c.q, c.k, c.pos, c.table, c.axes, interleaved)
    normed = lnmod.qknorm_rotary_forward(c.q, c.k, c.wq, c.wk, c.pos, c.table, c.axes, interleaved)
    pos = c.pos.clone()
    pos[1, 5, 1] = bad
    f = axis_features(c.axes, interleaved, 1).cuda()
    for got, ref in zip(lnmod.rotary(c.q, c.k, pos, c.table, c.axes, interleaved), want):
        assert bool(got[1, 5][:, f].isnan().all())
        rest = got.clone()
        rest[1, 5, :, f] = ref[1, 5, :, f]
        assert torch.equal(rest, ref)
    for got, ref in zip(lnmod.qknorm_rotary_forward(c.q, c.k, c.wq, c.wk, pos, c.table, c.axes, interleaved)[:2], normed):
        assert bool(got[1, 5][:, f].isnan().all())
        rest = got.clone()
        rest[1, 5, :, f] = ref[1, 5, :, f]
        assert torch.equal(rest, ref)
    # backwards the token's row of gradients, and through it the weights'
    args = (c.q, c.k, c.wq, c.wk, *normed[2:])
    ref = lnmod.qknorm_rotary_backward(c.dq, c.dk, *args, c.pos, c.table, c.axes, interleaved)
    got = lnmod.qknorm_rotary_backward(c.dq, c.dk, *args, pos, c.table, c.axes, interleaved)
    for g, r in zip(got[:2], ref):
        assert bool(g[1, 5].isnan().all())
        g = g.clone()
        g[1, 5] = r[1, 5]
        assert torch.equal(g, r)
    for g, r, n in zip(got[2:], ref[2:], (6, 2)):
        hit = torch.zeros(n, 72, dtype=torch.bool, device="cuda")
        hit[:, f] = True
        assert bool(g.view(n, 72)[hit].isnan().all()) and torch.equal(g.view(n, 72)[~hit], r.view(n, 72)[~hit])


@BOTH
@PAIRS
@pytest.mark.parametrize("hd,axes,heads", [(8, (8,), (3, 1)), (40, (16, 16), (5, 5)), (72, (24, 24), (2, 7)), (128, (44, 42, 10), (33, 9))],
                         ids=str)
def test_values_that_are_no_numbers_stay_where_they_are(hd, axes, heads, interleaved, dtype):
    c = Case(dtype, lead=(3, 19), heads=heads, hd=hd, axes=axes, interleaved=interleaved)
    R = sum(axes)
    q = c.q.clone()
    marks = [(0, 0, 0, 0, float("nan")), (1, 7, heads[0] - 1, R - 1, float("inf")), (2, 18, heads[0] // 2, hd - 1, float("-inf"))]
    for b, s, h, d, v in marks:
        q[b, s, h, d] = v
    want, _ = lnmod.rotary(c.q, c.k, c.pos, c.table, c.axes, interleaved)
    got, _ = lnmod.rotary(q, c.k, c.pos, c.table, c.axes, interleaved)
    hit = torch.zeros_like(got, dtype=torch.bool)
    for b, s, h, d, v in marks:
        if d >= R:
            assert float(got[b, s, h, d]) == v
            hit[b, s, h, d] = True
            continue
        other = (d ^ 1) if interleaved else (d + R // 2) % R
        assert not bool(got[b, s, h, d].isfinite()) or not bool(got[b, s, h, other].isfinite())
        hit[b, s, h, d] = hit[b, s, h, other] = True
    assert torch.equal(got[~hit], want[~hit])
    # with the norm: the token's row, or the head
    for per_head in (False, True):
        wq, wk = (torch.ones(hd if per_head else n * hd, dtype=dtype, device="cuda") for n in heads)
        want = lnmod.qknorm_rotary_forward(c.q, c.k, wq, wk, c.pos, c.table, c.axes, interleaved)
        got = lnmod.qknorm_rotary_forward(q, c.k, wq, wk, c.pos, c.table, c.axes, interleaved)
        assert same(got[1], want[1]) and same(got[3], want[3])
        hit = torch.zeros_like(got[0], dtype=torch.bool)
        for b, s, h, d, v in marks:
            part = (b, s, h) if per_head else (b, s)
            hit[part] = True
            assert not bool(got[0][part].isfinite().all())
            assert not float(got[2][part]) > 0                              # 1 / root: 0 or NaN
        assert torch.equal(got[0][~hit], want[0][~hit])
        ref = lnmod.qknorm_rotary_backward(c.dq, c.dk, c.q, c.k, wq, wk, *want[2:], c.pos, c.table, c.axes, interleaved)
        out = lnmod.qknorm_rotary_backward(c.dq, c.dk, q, c.k, wq, wk, *got[2:], c.pos, c.table, c.axes, interleaved)
        assert torch.equal(out[0][~hit], ref[0][~hit]) and same(out[1], ref[1]) and same(out[3], ref[3])
        assert not bool(out[2].isfinite().all())


@BOTH
@pytest.mark.parametrize("per_head", [False, True], ids=["row", "head"])
def test_rows_of_zeros(per_head, dtype):
    c = Case(dtype, lead=(2, 21), heads=(4, 3), hd=64, axes=(16, 24, 24), per_head=per_head)
    c.q[0, 3] = 0
    c.k[1, 20] = 0
    out = lnmod.qknorm_rotary_forward(c.q, c.k, c.wq, c.wk, c.pos, c.table, c.axes, True, EPS)
    assert bool((out[0][0, 3] == 0).all()) and bool((out[1][1, 20] == 0).all())
    assert torch.allclose(out[2][0, 3].cpu(), torch.tensor(1e3), rtol=2.0 ** -20)
    dq, dk, dwq, dwk = lnmod.qknorm_rotary_backward(c.dq, c.dk, c.q, c.k, c.wq, c.wk, *out[2:], c.pos, c.table, c.axes)
    c.check_backward(dq, dwq.to(dtype), c.q, c.wq, c.dq, "q")
    c.check_backward(dk, dwk.to(dtype), c.k, c.wk, c.dk, "k")


@BOTH
@PAIRS
def test_what_lies_between_and_behind_is_left_alone(interleaved, dtype):
    """Inputs in the middle of NaNs are read alone; dense outputs in the middle of sevens are written alone."""
    B, S, heads, hd, axes = 2, 23, (5, 3), 72, (24, 24, 24)
    c = Case(dtype, lead=(B, S), heads=heads, hd=hd, axes=axes, interleaved=interleaved)
    code, kind = (lnmod.LNMOD_BF16, bf) if dtype == bf else (lnmod.LNMOD_F32, torch.float32)
    rot = lnmod.Rotation(c.pos.data_ptr(), S, c.table.data_ptr(), c.table.shape[0], 3, (24, 24, 24, 0), int(interleaved))
    st = torch.cuda.current_stream().cuda_stream
    keep = []

    def spread(t):
        big = torch.full((B + 1, S + 2, t.shape[2] + 2, hd + 8), float("nan"), dtype=kind, device="cuda")
        view = big[:B, 1:S + 1, 1:-1, :hd]
        view.copy_(t)
        keep.append(big)
        return lnmod.Heads(view.data_ptr(), *view.stride()[:3])

    def fenced(n, dt=kind):
        big = torch.full((n + 512,), 7.0, dtype=dt, device="cuda")
        keep.append(big)
        return big, big[256:256 + n]

    def intact(big, n):
        return bool((big[:256] == 7).all()) and bool((big[256 + n:] == 7).all())

    x = [spread(t) for t in (c.q, c.k)]
    g = [spread(t) for t in (c.dq, c.dk)]
    n = [t.numel() for t in (c.q, c.k)]
    outs = [fenced(k) for k in n]
    assert lnmod.lnmod_rotary(x[0], x[1], B, S, *heads, hd, rot, 0, st, *(o[1].data_ptr() for o in outs), code) == 0
    want = lnmod.rotary(c.q, c.k, c.pos, c.table, axes, interleaved)
    for (big, at), k, w in zip(outs, n, want):
        assert torch.equal(at.view_as(w), w) and intact(big, k)
    for per_head in (0, 1):
        wq, wk = (torch.rand(hd if per_head else h * hd, device="cuda").to(kind) for h in heads)
        ref = lnmod.qknorm_rotary_forward(c.q, c.k, wq, wk, c.pos, c.table, axes, interleaved)
        rs = [fenced(B * S * (h if per_head else 1), torch.float32) for h in heads]
        outs = [fenced(k) for k in n]
        assert lnmod.lnmod_qknorm_rotary_forward(x[0], x[1], wq.data_ptr(), wk.data_ptr(), B, S, *heads, hd, rot, 1e-6, per_head, st,
                                                 *(o[1].data_ptr() for o in outs + rs), code) == 0
        for (big, at), w in zip(outs + rs, ref):
            assert torch.equal(at.view_as(w), w) and intact(big, w.numel())
        ref = lnmod.qknorm_rotary_backward(c.dq, c.dk, c.q, c.k, wq, wk, *ref[2:], c.pos, c.table, axes, interleaved)
        size = lnmod.lnmod_qknorm_rotary_backward_workspace_bytes(B * S, *heads, hd, per_head)
        ws = fenced(size // 4, torch.float32)
        outs = [fenced(k) for k in n] + [fenced(w.numel(), torch.float32) for w in (wq, wk)]
        assert lnmod.lnmod_qknorm_rotary_backward(g[0], g[1], x[0], x[1], wq.data_ptr(), wk.data_ptr(), B, S, *heads, hd, rot, per_head,
                                                  st, rs[0][1].data_ptr(), rs[1][1].data_ptr(), *(o[1].data_ptr() for o in outs),
                                                  ws[1].data_ptr(), size, code, 0) == 0
        for (big, at), w in zip(outs, ref):
            assert torch.equal(at.view_as(w), w) and intact(big, w.numel())
        assert intact(ws[0], size // 4)


@pytest.mark.parametrize("lead", [(0,), (0, 5), (2, 0)], ids=str)
@BOTH
def test_no_tokens(lead, dtype):
    q, k = torch.empty(*lead, 4, 64, dtype=dtype, device="cuda"), torch.empty(*lead, 2, 64, dtype=dtype, device="cuda")
    wq, wk = torch.ones(256, dtype=dtype, device="cuda"), torch.ones(128, dtype=dtype, device="cuda")
    pos, table = torch.empty(lead[-1], 1, dtype=torch.int32, device="cuda"), lnmod.rotary_table(3, (64,))
    leaves = [t.requires_grad_() for t in (q, k, wq, wk)]
    ys = F.rotary(q, k, pos, table, (64,))
    assert [y.shape for y in ys] == [q.shape, k.shape]
    torch.autograd.grad(ys, (q, k), ys)
    ys = F.qk_norm_rotary(*leaves, pos, table, (64,))
    grads = torch.autograd.grad(ys, leaves, ys)
    assert [g.shape for g in grads] == [t.shape for t in leaves] and bool((grads[2] == 0).all()) and bool((grads[3] == 0).all())


@PAIRS
def test_beyond_four_gigabytes(interleaved):
    """The first, middle and last tokens are what they are by themselves."""
    S, H, hd, axes = 470000, 40, 128, (44, 42, 42)                             # 4.8 GB
    table = lnmod.rotary_table(64, axes)
    pos = torch.randint(0, 64, (S, 3), dtype=torch.int32, device="cuda")
    q = torch.randn(1000, H, hd, device="cuda").to(bf).repeat(S // 1000, 1, 1)
    q[-7:] = torch.randn(7, H, hd, device="cuda").to(bf)
    w = torch.rand(H * hd, device="cuda").to(bf)
    dy = q.flip(0)
    parts = [slice(0, 3), slice(S // 2, S // 2 + 5), slice(S - 7, S)]
    y = lnmod.rotary(q, None, pos, table, axes, interleaved)[0]
    for p in parts:
        assert torch.equal(y[p], lnmod.rotary(q[p].clone(), None, pos[p].clone(), table, axes, interleaved)[0])
    del y
    for ww in (w, w[:hd].clone()):
        y, z, rq, rk = lnmod.qknorm_rotary_forward(q, q, ww, ww, pos, table, axes, interleaved)
        dq, dk, dwq, dwk = lnmod.qknorm_rotary_backward(dy, dy, q, q, ww, ww, rq, rk, pos, table, axes, interleaved)
        assert torch.equal(y, z) and torch.equal(dq, dk) and torch.equal(dwq, dwk)
        for p in parts:
            part = q[p].clone()
            one = lnmod.qknorm_rotary_forward(part, part, ww, ww, pos[p].clone(), table, axes, interleaved)
            assert torch.equal(y[p], one[0]) and torch.equal(rq[p], one[2])
            back = lnmod.qknorm_rotary_backward(dy[p].clone(), dy[p].clone(), part, part, ww, ww, one[2], one[3], pos[p].clone(), table,
                                                axes, interleaved)
            assert torch.equal(dq[p], back[0])
        del y, z, dq, dk
    # heads in front of the tokens: a head's stride is beyond 32 bits with a view of few tokens at the end
    far = torch.zeros(2, S * H, hd, dtype=bf, device="cuda")[:, -9:].transpose(0, 1)
    far.copy_(q[-9:, :2])
    assert far.stride(1) * 2 > 1 << 32
    got = lnmod.rotary(far, None, pos[-9:].clone(), table, axes, interleaved)[0]
    assert torch.equal(got, lnmod.rotary(q[-9:, :2].clone(), None, pos[-9:].clone(), table, axes, interleaved)[0])


# Heads that take 1 to 57 rounds of a wave's lanes, with idle lanes and without: one to eight units a lane, one to eight waves a
# token, two tokens a block, tokens side by side in a wave, heads in pieces for different blocks.
MANY = [(128, (4, 3)), (128, (8, 5)), (128, (12, 12)), (128, (17, 16)), (128, (28, 4)), (128, (36, 20)), (128, (52, 8)), (128, (64, 41)),
        (72, (113, 60)), (72, (29, 97)), (40, (200, 3)), (256, (32, 7)), (8, (1000, 33)), (24, (65, 341)), (136, (60, 1))]


@BOTH
@pytest.mark.parametrize("shape", MANY, ids=str)
def test_every_launch_shape(shape, dtype):
    hd, heads = shape
    R = hd // 16 * 16 or 8
    for interleaved, tokens in ((True, 53), (False, 700)):
        for per_head in (False, True):
            c = Case(dtype, lead=(tokens,), heads=heads, hd=hd, axes=(R // 2, R // 2), interleaved=interleaved, per_head=per_head)
            yq, yk, rq, rk = lnmod.qknorm_rotary_forward(c.q, c.k, c.wq, c.wk, c.pos, c.table, c.axes, interleaved, EPS)
            c.check_forward(yq, c.q, c.wq, "q")
            c.check_forward(yk, c.k, c.wk, "k")
            dq, dk, dwq, dwk = lnmod.qknorm_rotary_backward(c.dq, c.dk, c.q, c.k, c.wq, c.wk, rq, rk, c.pos, c.table, c.axes, interleaved)
            c.check_backward(dq, dwq, c.q, c.wq, c.dq, "q")
            c.check_backward(dk, dwk, c.k, c.wk, c.dk, "k")
        for y, x in zip(lnmod.rotary(c.q, c.k, c.pos, c.table, c.axes, interleaved), (c.q, c.k)):
            x = x.double().cpu()
            near(y.cpu(), c.turn(x), 4 * U * c.turn(x, magnitude=True), "rotation")


@BOTH
def test_more_heads_than_a_norm_takes(dtype):
    """Rotation, and the norm over heads, of rows beyond 8192 features, in pieces."""
    c = Case(dtype, lead=(31,), heads=(1000, 77), hd=128, axes=(44, 42, 42), per_head=True)
    for y, x in zip(lnmod.rotary(c.q, c.k, c.pos, c.table, c.axes), (c.q, c.k)):
        x = x.double().cpu()
        near(y.cpu(), c.turn(x), 4 * U * c.turn(x, magnitude=True), "rotation")
    yq, yk, rq, rk = lnmod.qknorm_rotary_forward(c.q, c.k, c.wq, c.wk, c.pos, c.table, c.axes, True, EPS)
    c.check_forward(yq, c.q, c.wq, "q")
    dq, dk, dwq, dwk = lnmod.qknorm_rotary_backward(c.dq, c.dk, c.q, c.k, c.wq, c.wk, rq, rk, c.pos, c.table, c.axes)
    c.check_backward(dq, dwq, c.q, c.wq, c.dq, "q")
    c.check_backward(dk, dwk, c.k, c.wk, c.dk, "k")
    w = torch.ones(128 * 1000, dtype=dtype, device="cuda")
    with pytest.raises(lnmod.LnmodError, match="unsupported"):
        lnmod.qknorm_rotary_forward(c.q, c.k, w, w[:77 * 128], c.pos, c.table, c.axes)


@BOTH
def test_one_tensor_and_one_pair(dtype):
    """k None with its gradient; two features turned by a table of one row; a position of its own for every token."""
    c = Case(dtype, lead=(3, 21), heads=(5, 2), hd=40, axes=(2,), rows=1, shared=False)
    q = c.q.detach().requires_grad_()
    y = F.rotary(q, None, c.pos, c.table, c.axes)
    d, = torch.autograd.grad(y, q, c.dq)
    z = F._Rotary.apply(q, None, c.pos, c.table, c.axes, True)
    e, = torch.autograd.grad(z, q, c.dq)
    assert torch.equal(y, z) and torch.equal(d, e)
    assert torch.equal(y, c.q) and torch.equal(d, c.dq)                         # position 0 turns nothing
    c = Case(dtype, lead=(3, 21), heads=(5, 2), hd=40, axes=(2,), shared=False)
    for y, x in zip(lnmod.rotary(c.q, c.k, c.pos, c.table, c.axes, inverse=True), (c.q, c.k)):
        x = x.double().cpu()
        near(y.cpu(), c.turn(x, back=True), 4 * U * c.turn(x, magnitude=True), "one pair")


@BOTH
def test_repeated_samples_and_heads(dtype):
    """Expanded inputs: a stride of 0.  Their gradients are sums over the copies: of three in float32 and one rounding, or three
    roundings in bf16 (torch adds them)."""
    c = Case(dtype, lead=(3, 17), heads=(4, 4), hd=64)
    one = c.q[:1].detach().requires_grad_()
    head = c.k[:, :, :1].detach().requires_grad_()
    q, k = one.expand(3, -1, -1, -1), head.expand(-1, -1, 4, -1)
    got = F.qk_norm_rotary(q, k, c.wq, c.wk, c.pos, c.table, c.axes)
    want = F.qk_norm_rotary(q.detach().clone(), k.detach().clone(), c.wq, c.wk, c.pos, c.table, c.axes)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    grads = torch.autograd.grad(got, (one, head), (c.dq, c.dk))
    lq, lk = (t.detach().clone().requires_grad_() for t in (q, k))
    whole = torch.autograd.grad(F.qk_norm_rotary(lq, lk, c.wq, c.wk, c.pos, c.table, c.axes), (lq, lk), (c.dq, c.dk))
    for g, w, dim in ((grads[0], whole[0], 0), (grads[1], whole[1], 2)):
        w = w.double()
        tol = 4 * torch.finfo(dtype).eps / 2 * w.abs().sum(dim, keepdim=True)
        assert bool(((g.double() - w.sum(dim, keepdim=True)).abs() <= tol).all())


# ---- gradients against differences ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("per_head", [False, True], ids=["row", "head"])
@PAIRS
def test_gradients_against_differences(interleaved, per_head):
    """Along a direction d as long as the row that it is added to, y(t) = T((x + t d) r(t) w) has its nearest singularities at
    |t| = 1.  On |t| = 1/2 both factors of the root are at least 1/2, so a normed value is at most 2 (|x| + |d| / 2) r |w| and a turned
    one the sum of two, M: coefficients of the series are below M 2^k.  (8 (f(h) - f(-h)) - (f(2h) - f(-2h))) / 12 h is off by
    the sum over odd k >= 5 of M 2^k h^(k-1) (2^(k+1) - 16) / 12 < 180 h^4 M, and by 18 / 12 h times the error of a value, 2^-17 of the
    pair's magnitude; the gradient's own error is 2^-16 of the sum of magnitudes."""
    c = Case(torch.float32, lead=(2, 9), heads=(3, 2), hd=40, axes=(16, 24), interleaved=interleaved, per_head=per_head)
    over = (-1,) if per_head else (-2, -1)
    h = 2.0 ** -5
    g = torch.Generator(device="cuda").manual_seed(8)

    def forward(q, k, wq, wk):
        return [t.double() for t in lnmod.qknorm_rotary_forward(q, k, wq, wk, c.pos, c.table, c.axes, interleaved, EPS)[:2]]

    def direction(x):
        d = torch.randn(x.shape, generator=g, device="cuda")
        return d * (x.square().sum(over, keepdim=True) / d.square().sum(over, keepdim=True)).sqrt()

    dirs = [direction(c.q), direction(c.k)]
    fwd = lnmod.qknorm_rotary_forward(c.q, c.k, c.wq, c.wk, c.pos, c.table, c.axes, interleaved, EPS)
    grads = lnmod.qknorm_rotary_backward(c.dq, c.dk, c.q, c.k, c.wq, c.wk, *fwd[2:], c.pos, c.table, c.axes, interleaved)
    at = [forward(c.q + t * h * dirs[0], c.k + t * h * dirs[1], c.wq, c.wk) for t in (1, -1, 2, -2)]
    for i, (x, d, dy, w, n) in enumerate(zip((c.q, c.k), dirs, (c.dq, c.dk), (c.wq, c.wk), (3, 2))):
        slope = (8 * (at[0][i] - at[1][i]) - (at[2][i] - at[3][i])) / (12 * h)
        got = (grads[i].double() * d.double()).sum(over)
        want = (slope * dy.double()).sum(over)
        rms = (x.double().square().mean(over, keepdim=True) + EPS).sqrt()
        size = (x.double().abs() + 0.5 * d.double().abs()).amax(over, keepdim=True) / rms * float(w.abs().max())
        M = 2 * 2 * size                                                       # a turned value: at most the sum of two
        bound = (dy.double().abs() * (180 * h ** 4 * M + 1.5 / h * 2.0 ** -17 * M)).sum(over)
        bound = bound + 2.0 ** -16 * (dy.double().abs().sum(over) * 8 * size.squeeze(over))
        assert bool(((got - want).abs() <= bound).all())
        assert float(bound.max()) < 0.5 * float(want.abs().max())
    # the weights: y is linear in them
    dirs = [torch.randn(w.shape, generator=g, device="cuda") for w in (c.wq, c.wk)]
    up, down = (forward(c.q, c.k, c.wq + s * dirs[0], c.wk + s * dirs[1]) for s in (0.5, -0.5))
    for i, (dy, x) in enumerate(((c.dq, c.q), (c.dk, c.k))):
        got, want = (grads[2 + i].double() * dirs[i].double()).sum(), ((up[i] - down[i]) * dy.double()).sum()
        bound = 2.0 ** -14 * (dy.double().abs() * (up[i].abs() + down[i].abs() + 4 * x.double().abs().amax() * float(dirs[i].abs().max()))).sum()
        assert abs(float(got - want)) <= float(bound)


@BOTH
@PAIRS
def test_the_gradient_is_the_rotation_of_a_difference(interleaved, dtype):
    """A rotation keeps lengths, and turning back undoes it: each rounding is half a step of at most sqrt(2) of the value's pair."""
    c = Case(dtype, lead=(3, 50), heads=(7, 3), hd=64, axes=(16, 24, 24), interleaved=interleaved)
    y, _ = lnmod.rotary(c.q, c.k, c.pos, c.table, c.axes, interleaved)
    back, _ = lnmod.rotary(y, c.k, c.pos, c.table, c.axes, interleaved, inverse=True)
    pair = c.turn(c.q.double().cpu(), magnitude=True)
    # y off by e = (half a step + 8 u) of the pair in each of its two values; turned back that is 2 e; and once more itself
    tol = 3.1 * (torch.finfo(dtype).eps / 2 + 8 * U) * pair
    assert bool(((back.double() - c.q.double()).cpu().abs() <= tol).all())


# ---- host paths, transforms, hooks ----------------------------------------------------------------------------------------
CALLS = {"rotary": (lambda c: (c.q, c.k), lambda c, *t: F.rotary(*t, c.pos, c.table, c.axes, c.interleaved),
                    lambda c, *t: F._Rotary.apply(*t, c.pos, c.table, c.axes, c.interleaved)),
         "norm": (lambda c: (c.q, c.k, c.wq, c.wk), lambda c, *t: F.qk_norm_rotary(*t, c.pos, c.table, c.axes, c.interleaved, EPS),
                  lambda c, *t: F._QkNormRotary.apply(*t, c.pos, c.table, c.axes, c.interleaved, EPS))}


@BOTH
@pytest.mark.parametrize("op", sorted(CALLS))
@pytest.mark.parametrize("layout", ["dense", "fused"])
def test_the_native_host_path_and_the_python_path_agree(layout, op, dtype):
    """Outputs and gradients bit for bit, also where one output has no gradient, where saved tensors go through hooks, and where
    gradients come in layouts that the kernels do not read."""
    c = Case(dtype, lead=(2, 37), heads=(6, 2), hd=72, axes=(16, 24, 16), layout=layout)
    inputs, native, python = CALLS[op]
    ts = [t.detach().requires_grad_() for t in inputs(c)]
    odd = torch.randn(2, 37, 6, 73, device="cuda").to(dtype)[..., 1:]            # rows of 73 at an odd element

    def results(call, how):
        outs = call(c, *ts)
        if how == "both":
            grads = torch.autograd.grad(outs, ts, (c.dq, c.dk))
        elif how == "one":
            grads = torch.autograd.grad(outs[1], ts, c.dk, allow_unused=True)
        elif how == "sum":
            grads = torch.autograd.grad(outs[0].float().sum() + outs[1].sum(), ts)
        else:
            grads = torch.autograd.grad(outs, ts, (odd, c.dk.flip(1).transpose(1, 2).contiguous().transpose(1, 2)))
        return [o.detach() for o in outs] + [torch.zeros_like(t) if g is None else g for g, t in zip(grads, ts)], outs

    for how in ("both", "one", "sum", "odd"):
        a, outs = results(native, how)
        b, ref = results(python, how)
        assert type(outs[0].grad_fn) is not type(ref[0].grad_fn) and len(a) == len(b)
        assert all(same(u, v) for u, v in zip(a, b)), how
        with torch.autograd.graph.save_on_cpu():
            assert all(same(u, v) for u, v in zip(results(native, how)[0], results(python, how)[0]))
    # an input alone
    for k in range(len(ts)):
        only = [t.detach().requires_grad_(i == k) for i, t in enumerate(ts)]
        outs = native(c, *only)
        whole = torch.autograd.grad(native(c, *ts), ts, (c.dq, c.dk))
        used = [(o, d) for o, d in zip(outs, (c.dq, c.dk)) if o.requires_grad]
        got, = torch.autograd.grad([o for o, _ in used], only[k], [d for _, d in used])
        assert same(got, whole[k])
    leaves = [t.detach().requires_grad_() for t in inputs(c)]
    for _ in range(2):
        torch.autograd.backward(native(c, *leaves), (c.dq, c.dk))
    for t, g in zip(leaves, torch.autograd.grad(native(c, *leaves), leaves, (c.dq, c.dk))):
        assert same(t.grad, g + g)


@pytest.mark.parametrize("op", sorted(CALLS))
def test_transforms_are_refused(op):
    c = Case(torch.float32)
    inputs, native, _ = CALLS[op]
    ts = inputs(c)
    with pytest.raises(RuntimeError):
        torch.func.vmap(lambda t: native(c, t, *ts[1:])[0])(ts[0][None])
    with pytest.raises(RuntimeError):
        torch.func.grad(lambda t: native(c, t, *ts[1:])[0].sum())(ts[0])
    with torch.autograd.forward_ad.dual_level(), pytest.raises(RuntimeError):
        native(c, torch.autograd.forward_ad.make_dual(ts[0], ts[0]), *ts[1:])
    leaf = ts[0].clone().requires_grad_()
    dy = torch.randn_like(leaf).requires_grad_()
    first, = torch.autograd.grad(native(c, leaf, *ts[1:])[0], leaf, dy, create_graph=True)
    assert not first.requires_grad                                             # no half-connected second derivative
    codes, scales = lnmod.quantize_rows(torch.randn(4, 64, device="cuda"))
    with pytest.raises(RuntimeError):
        torch.func.vmap(lambda t: lnmod.code_product(t, scales, codes, scales))(codes[None])


def test_native_and_python_bindings_agree():
    raw = torch.cuda.current_stream().cuda_stream
    c = Case(bf, lead=(2, 33), heads=(6, 2), hd=64, layout="fused")
    args = (c.pos, c.table, c.axes, c.interleaved)
    for inverse in (False, True):
        for k in (c.k, None):
            a, b = (lnmod.rotary(c.q, k, *args, inverse=inverse, stream=s) for s in (None, raw))
            assert all((u is None and v is None) or torch.equal(u, v) for u, v in zip(a, b)) and len(a) == len(b)
    a, b = (lnmod.qknorm_rotary_forward(c.q, c.k, c.wq, c.wk, *args, stream=s) for s in (None, raw))
    assert all(torch.equal(u, v) for u, v in zip(a, b))
    ws = torch.empty(lnmod.lnmod_qknorm_rotary_backward_workspace_bytes(66, 6, 2, 64, 0), dtype=torch.uint8, device="cuda")
    back = [lnmod.qknorm_rotary_backward(c.dq, c.dk, c.q, c.k, c.wq, c.wk, *a[2:], *args, **kw) for kw in ({}, dict(stream=raw, ws=ws))]
    assert all(torch.equal(u, v) for u, v in zip(*back))
    x = torch.randn(5, 7, 136, device="cuda").to(bf)
    for code in ("int8", "e4m3"):
        p, q = (lnmod.quantize_rows(x, code, stream=s) for s in (None, raw))
        assert all(torch.equal(u.float(), v.float()) for u, v in zip(p, q))
        w, sw = lnmod.quantize_rows(torch.randn(24, 136, device="cuda"), code)
        for bias in (None, torch.randn(24, device="cuda")):
            y, z = (lnmod.code_product(*p, w, sw, bias, torch.float32, stream=s) for s in (None, raw))
            assert torch.equal(y, z)


def test_a_handle_of_zero_is_the_default_stream():
    side = torch.cuda.Stream()
    for around in (torch.cuda.default_stream(), side):
        with torch.cuda.stream(around):
            with lnmod._on_stream(0) as handle:
                assert handle == 0 and torch.cuda.current_stream() == torch.cuda.default_stream()
            with lnmod._on_stream(side.cuda_stream) as handle:
                assert handle == side.cuda_stream
            with lnmod._on_stream(None) as handle:
                assert handle == around.cuda_stream


# ---- used together ----------------------------------------------------------------------------------------------------------
HEADS, KV, HD, AXES = 6, 2, 64, (16, 24, 24)


def block_inputs(seed=1, B=2, grid=(3, 7, 5), D=512):
    g = torch.Generator(device="cuda").manual_seed(seed)
    S = grid[0] * grid[1] * grid[2]

    def make(*shape, std=1.0, mean=0.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(bf)

    s = dict(x=make(B, S, D), w=make(D, mean=1.0, std=0.1), proj=make((HEADS + 2 * KV) * HD, D, std=D ** -0.5),
             bias=make((HEADS + 2 * KV) * HD), out=make(D, HEADS * HD, std=0.05), wq=make(HEADS * HD, mean=1.0, std=0.1),
             wk=make(KV * HD, mean=1.0, std=0.1), dq=make(B, HEADS, S, HD).transpose(1, 2), dk=make(B, S, KV, HD))
    s["pos"], s["table"] = lnmod.rotary_grid(*grid), lnmod.rotary_table(max(grid), AXES)
    return s


def block(s, code="int8"):
    """What stands before a layer's attention, in serving: norm with codes, the fused projection of codes, norm and rotation on its
    output in place of copies of q and k; then the step back through norm and rotation, and the output's projection."""
    proj, proj_scales = lnmod.quantize_rows(s["proj"], code)
    codes, scales = lnmod.rmsnorm_quant_forward(s["x"], s["w"], None, 1e-6, code, 0)[:2]
    qkv = lnmod.code_product(codes, scales, proj, proj_scales, s["bias"])
    q = qkv[..., :HEADS * HD].unflatten(-1, (HEADS, HD)).requires_grad_()
    k = qkv[..., HEADS * HD:(HEADS + KV) * HD].unflatten(-1, (KV, HD)).requires_grad_()
    wq, wk = (s[n].detach().requires_grad_() for n in ("wq", "wk"))
    ys = F.qk_norm_rotary(q, k, wq, wk, s["pos"], s["table"], AXES)
    grads = torch.autograd.grad(ys, (q, k, wq, wk), (s["dq"], s["dk"]))
    plain = F.rotary(q.detach(), k.detach(), s["pos"], s["table"], AXES, False)
    o = ys[0].detach().flatten(-2)
    oc, os_ = lnmod.quantize_rows(o, code)
    ow, ows = lnmod.quantize_rows(s["out"], code)
    y = lnmod.code_product(oc, os_, ow, ows)
    return [codes.float(), scales, qkv, ys[0].detach(), ys[1].detach(), *grads, *plain, oc.float(), os_, y]


@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_a_run_of_them_together(code):
    """Each link against the formula on what the link before it gave."""
    s = block_inputs()
    got = block(s, code)
    codes, scales, qkv, yq, yk, dq, dk, dwq, dwk, pq, pk, oc, os_, y = got
    proj, ps = (t.float() for t in lnmod.quantize_rows(s["proj"], code))
    ow, ows = (t.float() for t in lnmod.quantize_rows(s["out"], code))

    def product(a, sa, w, sw, b):
        a, sa, w, sw = (t.cpu().double() for t in (a, sa, w, sw))
        v = (a @ w.t()) * sa[..., None] * sw
        bias = 0 if b is None else b.cpu().double()
        slack = 4 * U * (v.abs() + abs(bias))
        if code == "e4m3":       # eight products are aligned to 2^-13 of the largest; the rest as in float32
            K = a.shape[-1]
            each = sum((a[..., None, k:k + 8] * w[:, k:k + 8]).abs().amax(-1) for k in range(0, K, 8))
            slack = slack + (7 * 2.0 ** -13 * each + K * U * (a.abs() @ w.abs().t())) * sa[..., None] * sw
        return v + bias, slack

    want, slack = product(codes, scales, proj, ps, s["bias"])
    near(qkv.cpu(), want, slack, "qkv")
    c = Case.__new__(Case)
    c.axes, c.interleaved, c.per_head, c.hd, c.pos = AXES, True, False, HD, s["pos"]
    q, k = qkv[..., :HEADS * HD].unflatten(-1, (HEADS, HD)), qkv[..., HEADS * HD:(HEADS + KV) * HD].unflatten(-1, (KV, HD))
    c.check_forward(yq, q, s["wq"], "q")
    c.check_forward(yk, k, s["wk"], "k")
    c.check_backward(dq, dwq, q, s["wq"], s["dq"], "q")
    c.check_backward(dk, dwk, k, s["wk"], s["dk"], "k")
    c.interleaved = False
    near(pq.cpu(), c.turn(q.double().cpu()), 4 * U * c.turn(q.double().cpu(), magnitude=True), "halves")
    want, slack = product(oc, os_, ow, ows, None)
    near(y.cpu(), want, slack, "y")
    for u, v in zip(got, block(s, code)):                                     # and twice the same bits
        assert torch.equal(u, v)


def test_another_stream():
    s = block_inputs(3)
    want = block(s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = block(s)
    side.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(want, got))
    c = Case(bf, lead=(2, 33), heads=(6, 2), hd=64)
    args = (c.pos, c.table, c.axes)
    ref = lnmod.qknorm_rotary_forward(c.q, c.k, c.wq, c.wk, *args)
    torch.cuda.synchronize()
    out = lnmod.qknorm_rotary_forward(c.q, c.k, c.wq, c.wk, *args, stream=side)
    back = lnmod.qknorm_rotary_backward(c.dq, c.dk, c.q, c.k, c.wq, c.wk, *out[2:], *args, stream=side)
    side.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(ref, out))
    assert all(torch.equal(u, v) for u, v in zip(back, lnmod.qknorm_rotary_backward(c.dq, c.dk, c.q, c.k, c.wq, c.wk, *ref[2:], *args)))


def test_two_graphs_with_eager_work_between_their_replays():
    sets = [block_inputs(5), block_inputs(6, B=1, grid=(2, 9, 13))]
    eager_before = [block(a) for a in sets]
    graphs, outs = [], []
    side = torch.cuda.Stream()
    for a in sets:
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            block(a)
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(block(a))
        graphs.append(g)
    for turn in range(4):
        for a in sets:
            a["x"].copy_(torch.randn(a["x"].shape, device="cuda"))
            a["dq"].copy_(torch.randn(a["dq"].shape, device="cuda"))
        eager = [block(a) for a in sets]
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        again = [block(a) for a in sets]
        torch.cuda.synchronize()
        for k in range(2):
            for u, v, z in zip(eager[k], outs[k], again[k]):
                assert torch.equal(u, v) and torch.equal(u, z)
            assert not torch.equal(eager[k][3], eager_before[k][3])


def test_calls_from_several_threads():
    """Each thread on a stream of its own, all at once: what one thread alone gives."""
    sets = [block_inputs(10 + k, grid=(3, 7, 5 + k)) for k in range(4)]
    want = [block(a) for a in sets]
    torch.cuda.synchronize()
    bad = []

    def work(k):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(6):
                    got = block(sets[k])
                    torch.cuda.current_stream().synchronize()
                    if not all(torch.equal(u, v) for u, v in zip(want[k], got)):
                        bad.append(k)
        except Exception as e:
            bad.append((k, e))

    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad
