"""The operators around attention in a block that is served in 8 bits and trained in bf16, case by case, for timing and
comparison: codes with one scale for a row, the product of such codes, rotary positions with several axes, and the query
and key norm with the rotation in the same pass.

A case is a dict of plain values.  `prepare` makes what a program holds before the call, `run` makes one pass (through the
package's entry points where `own` is true, else in elementary torch operations in 32 bits), `work` says what a pass cannot
do without, `exact` gives the same outputs from the definition in 64 bits.

Codes of a row v:
    amax = max |v|      s = fp32(max(amax, 2^-100) / Q)      r = fp32(1 / s)      Q = 127 (int8), 448 (e4m3)
    int8: code = v*r rounded to the nearest whole number, ties to even, one rounding
    e4m3: code = v*r rounded to fp32, then to the nearest e4m3, ties to even
Product:  y[m,n] = (sum_k a[m,k] w[n,k]) sa[m] sw[n] + bias[n]
Rotation: a head's first R features are R/2 pairs, shared out over the axes in order (axis a has axes[a] of the R features);
    pair i of an axis with d features turns by p * base^(-2i/d), p the token's position on that axis:
    (u, v) -> (u cos - v sin, u sin + v cos).  Pair j is the features 2j and 2j+1 (interleaved), or j and j + R/2.
Norm:     x * rsqrt(mean(x^2) + eps) * w over all features of a token, or over each head's, before the rotation.

Common keys:
  op        "rows"     lnmod.quantize_rows: codes and scales (serving), e4m3
            "product"  lnmod.code_product (serving)
            "rotary"   functional.rotary of q and k;  with step: and its gradients (training)
            "qk"       functional.qk_norm_rotary of q and k;  with step: and its gradients
  dtype     "bf16" or "f32" (product: of y);  code: "int8" or "e4m3"
  M, K, N   rows, features of a row, features of y (rows: M, K);  bias: whether the product adds one
  B, F, H, W            samples of F frames of H x W patches, one grid of positions for all of them;
  clips, clips_seed     or a packed batch of so many clips, each with a grid of its own
  heads, kv_heads, head_dim;  axes: features of time, height and width, as text;  interleaved;  per_head: the norm's width
  fused     q and k are views of one buffer that holds q, k and v of a token side by side (a fused projection's output)
  heads_first   the gradients arrive as views of [.., heads, tokens, features] (attention's layout)
"""
import math
import random

import torch

own = False

EPS = 1e-6
BASE = 10000.0
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LARGEST = {"int8": 127.0, "e4m3": 448.0}
SMALLEST = 2.0 ** -100


def listed():
    return [
        # One embedded timestep through a projection: the weights are all there is to read.
        dict(name="product_one_token", op="product", dtype="bf16", code="int8", M=1, K=5120, N=5120, bias=True),
        # A few dozen tokens (a text prompt) through a fused projection.
        dict(name="product_prompt", op="product", dtype="bf16", code="e4m3", M=96, K=4096, N=12288, bias=True),
        # Sizes that are no round numbers, fp32 results (logits, a small model).
        dict(name="product_ragged", op="product", dtype="f32", code="int8", M=1025, K=2600, N=1433, bias=False),
        # One still picture through the first half of a feed-forward block.
        dict(name="product_still", op="product", dtype="bf16", code="e4m3", M=8190, K=5120, N=13824, bias=True),
        # One clip through the fused projection of the 14B-shaped model: the largest product.
        dict(name="product_clip", op="product", dtype="bf16", code="int8", M=32760, K=5120, N=15360, bias=True),
        # The rows that such products read: a feed-forward block's inner activations, an odd number of them ...
        dict(name="rows_inner", op="rows", dtype="bf16", code="e4m3", M=1025, K=13824),
        # ... and one clip's tokens.
        dict(name="rows_clip", op="rows", dtype="bf16", code="e4m3", M=32760, K=5120),
        # Sampling: q and k of one long clip, views of the fused projection's output.
        dict(name="rotary_clip", op="rotary", step=False, dtype="bf16", B=1, F=21, H=45, W=80, heads=40, kv_heads=40,
             head_dim=128, axes="44,42,42", interleaved=True, fused=True, heads_first=False),
        # A toy model's step: fp32, fewer key heads, a part of the head turned, odd sizes.
        dict(name="rotary_toy_step", op="rotary", step=True, dtype="f32", B=3, F=3, H=13, W=17, heads=12, kv_heads=4,
             head_dim=64, axes="16,16,16", interleaved=False, fused=False, heads_first=True),
        # One new token.
        dict(name="qk_one_token", op="qk", step=False, dtype="bf16", B=1, F=1, H=1, W=1, heads=40, kv_heads=40, head_dim=128,
             axes="44,42,42", interleaved=True, per_head=False, fused=True, heads_first=False),
        # A training step of the 14B-shaped model, one clip, the norm over the whole projection.
        dict(name="qk_clip_step", op="qk", step=True, dtype="bf16", B=1, F=21, H=30, W=52, heads=40, kv_heads=40, head_dim=128,
             axes="44,42,42", interleaved=True, per_head=False, fused=False, heads_first=True),
        # Stills and clips packed, a norm per head, fewer key heads, halves turned.
        dict(name="qk_packed_step", op="qk", step=True, dtype="bf16", clips=24, clips_seed=5, heads=24, kv_heads=8, head_dim=96,
             axes="32,32,32", interleaved=False, per_head=True, fused=True, heads_first=False),
    ]


# A drawn case never does more than this (the listed ones: 5.2e12 operations, 3.1e9 bytes).
MOST_FLOPS = 4.5e12
MOST_BYTES = 2.8e9


def _spread(rng, lo, hi):
    """An integer from [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["product", "product", "rows", "rotary", "qk", "qk"])
    c = dict(op=op, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]))
    widths = [1152, 1536, 2048, 2560, 4096, 5120, 6144, 8960, 13824]
    if op in ("product", "rows"):
        c["code"] = "e4m3" if op == "rows" else rng.choice(["int8", "e4m3"])
        c["M"] = _spread(rng, 1, 32760)
        c["K"] = rng.choice(widths) if rng.random() < 0.6 else 8 * _spread(rng, 8, 2048)
        if op == "product":
            c["N"] = rng.choice(widths + [15360]) if rng.random() < 0.6 else _spread(rng, 16, 16384)
            c["bias"] = rng.random() < 0.6
            while work(c)["flops"] > MOST_FLOPS:
                c["M"] = c["M"] // 2 + 1
        return c
    c["step"] = rng.random() < 0.6
    head_dim, axes = rng.choice([(64, "16,24,24"), (64, "16,16,16"), (72, "24,24,24"), (96, "32,32,32"), (128, "44,42,42"),
                                 (128, "32,48,48"), (128, "16,56,56"), (128, "64,64"), (256, "64,96,96")])
    c.update(head_dim=head_dim, axes=axes, interleaved=rng.random() < 0.6, fused=rng.random() < 0.5,
             heads_first=rng.random() < 0.5)
    if sum(int(v) for v in axes.split(",")) % 8:
        c["interleaved"] = True
    c["heads"] = _spread(rng, 4, 48)
    if op == "qk":
        c["per_head"] = rng.random() < 0.5
        c["heads"] = min(c["heads"], 8192 // head_dim)
    c["kv_heads"] = c["heads"] if rng.random() < 0.6 else rng.randrange(1, c["heads"] + 1)
    if axes.count(",") == 2 and rng.random() < 0.4:
        c.update(clips=_spread(rng, 2, 32), clips_seed=rng.randrange(1 << 16))
    else:
        c.update(B=rng.choice([1, 1, 2, 3]), F=_spread(rng, 1, 21), H=_spread(rng, 1, 45), W=_spread(rng, 1, 80))
    while work(c)["bytes"] > MOST_BYTES:
        for k in ("clips", "F"):
            if k in c:
                c[k] = c[k] // 2 + (1 if c[k] > 1 else 0)
                break
        if c.get("F", 2) == 0 or (c.get("F") == 1 and work(c)["bytes"] > MOST_BYTES):
            c["F"], c["B"] = 1, 1
            c["H"] = c["H"] // 2 + 1
    return c


def _axes(case):
    return tuple(int(v) for v in case["axes"].split(","))


def _grids(case):
    """(frames, height, width) of each clip; one for all samples of a batch that is not packed."""
    if "clips" not in case:
        return [(case["F"], case["H"], case["W"])]
    rng = random.Random(case["clips_seed"])
    return [(1 if rng.random() < 0.5 else _spread(rng, 2, 9), _spread(rng, 9, 30), _spread(rng, 9, 52))
            for _ in range(case["clips"])]


def _tokens(case):
    """(rows of positions, tokens)"""
    n = sum(f * h * w for f, h, w in _grids(case))
    return n, n * case.get("B", 1)


def _positions(case):
    """[tokens, axes] of whole numbers, on the host."""
    parts = []
    for f, h, w in _grids(case):
        t, y, x = torch.meshgrid(torch.arange(f), torch.arange(h), torch.arange(w), indexing="ij")
        p = torch.stack([t, y, x], -1).reshape(-1, 3)
        parts.append(p if len(_axes(case)) == 3 else torch.stack([p[:, 0] * h + p[:, 1], p[:, 2]], -1))
    return torch.cat(parts)


def _frequencies(axes):
    """Of all pairs, in order: [R/2], float64."""
    return torch.cat([BASE ** (-torch.arange(0, d, 2, dtype=torch.float64) / d) for d in axes])


def prepare(case, seed):
    dt = DTYPES[case["dtype"]]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, mean=0.0, std=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(dt)

    def activations(*shape):
        # hidden states: off centre, wide, and one value in a thousand an outlier
        v = torch.randn(*shape, generator=g, device="cuda") * 2.0 + 0.5
        v *= torch.where(torch.rand(*shape, generator=g, device="cuda") < 1e-3, 50.0, 1.0)
        return v

    s = {"case": case}
    if case["op"] == "rows":
        s["x"] = activations(case["M"], case["K"]).to(dt)
        return s
    if case["op"] == "product":
        kind = torch.int8 if case["code"] == "int8" else torch.float8_e4m3fn
        q, s["scales"] = _row_codes(activations(case["M"], case["K"]), case["code"])
        s["codes"] = q.to(kind)
        q, s["w_scales"] = _row_codes(torch.randn(case["N"], case["K"], generator=g, device="cuda") * 0.02, case["code"])
        s["w"] = q.to(kind)
        s["bias"] = normal(case["N"], std=0.1) if case["bias"] else None
        return s
    heads, kv, hd, axes = case["heads"], case["kv_heads"], case["head_dim"], _axes(case)
    pos = _positions(case)
    # the program's plan: cosine and sine of every whole-numbered position it may meet, formed in 64 bits once
    angle = torch.arange(int(pos.max()) + 1, dtype=torch.float64).unsqueeze(1) * _frequencies(axes)
    s["table"] = torch.stack([angle.cos(), angle.sin()], -1).float().cuda()
    s["positions"] = pos.to(torch.int32).cuda()
    lead = (pos.shape[0],) if "clips" in case else (case["B"], pos.shape[0])
    if case["fused"]:
        both = normal(*lead, (heads + 2 * kv) * hd)
        s["q"] = both[..., :heads * hd].unflatten(-1, (heads, hd))
        s["k"] = both[..., heads * hd:(heads + kv) * hd].unflatten(-1, (kv, hd))
    else:
        s["q"], s["k"] = normal(*lead, heads, hd), normal(*lead, kv, hd)
    if case["op"] == "qk":
        s["wq"] = normal(hd if case["per_head"] else heads * hd, mean=1.0, std=0.1)
        s["wk"] = normal(hd if case["per_head"] else kv * hd, mean=1.0, std=0.1)
    if case["step"]:
        for name in ("q", "k", "wq", "wk"):
            if name in s:
                s[name] = s[name].detach().requires_grad_()
        for name, h in (("dq", heads), ("dk", kv)):
            if case["heads_first"]:
                s[name] = normal(*lead[:-1], h, lead[-1], hd).transpose(-2, -3)
            else:
                s[name] = normal(*lead, h, hd)
    return s


# ---- the plain forms -----------------------------------------------------------------------------------------------
def _row_codes(v, code):
    """fp32 values -> (fp32 values of the codes, scales).  The quotients, and the products of int8, are formed in 64 bits
    and rounded once (a division by a number on the host is a product with its rounded inverse)."""
    scales = (v.abs().amax(-1).clamp_min(SMALLEST).double() / LARGEST[code]).float()
    inv = (1.0 / scales.double()).float().unsqueeze(-1)
    if code == "int8":
        q = (v.double() * inv.double()).round().clamp(-127, 127).float()
    else:
        q = (v * inv).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).float()
    return q, scales


def _plain_product(s):
    y = (s["codes"].float() @ s["w"].float().t()) * s["scales"].unsqueeze(-1) * s["w_scales"]
    return (y if s["bias"] is None else y + s["bias"].float()).to(DTYPES[s["case"]["dtype"]])


def _cos_sin(s):
    """[positions, 1, R/2] each, fp32: the angles in 64 bits."""
    axes = _axes(s["case"])
    of = torch.cat([torch.full((d // 2,), a) for a, d in enumerate(axes)]).cuda()
    angle = s["positions"].double()[:, of] * _frequencies(axes).cuda()
    return angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)


def _turn(x, cos, sin, interleaved):
    R = 2 * cos.shape[-1]
    if interleaved:
        u, v = x[..., 0:R:2], x[..., 1:R:2]
    else:
        u, v = x[..., :R // 2], x[..., R // 2:R]
    a, b = u * cos - v * sin, u * sin + v * cos
    turned = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., R:]], -1)


def _plain_attention_input(s):
    case = s["case"]
    cos, sin = _cos_sin(s)
    ys, grads, weights = [], [], []
    for name in ("q", "k"):
        x = s[name].detach()
        dt, v = x.dtype, x.float()
        if case["op"] == "qk":
            over = -1 if case["per_head"] else (-2, -1)
            w = s["w" + name].detach().float()
            w = w if case["per_head"] else w.view(x.shape[-2:])
            rstd = 1.0 / (v.square().mean(over, keepdim=True) + EPS).sqrt()
            xhat = v * rstd
            v = xhat * w
        ys.append(_turn(v, cos, sin, case["interleaved"]).to(dt))
        if not case["step"]:
            continue
        g = _turn(s["d" + name].float(), cos, -sin, case["interleaved"])
        if case["op"] == "qk":
            dw = (g * xhat).flatten(0, -3).sum(0)
            weights.append((dw.sum(0) if case["per_head"] else dw.flatten()).to(dt))
            g = g * w
            g = (g - xhat * (g * xhat).mean(over, keepdim=True)) * rstd
        grads.append(g.to(dt))
    return tuple(ys + grads + weights)


# ---- one pass --------------------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if own:
        from paper_2605_17923_amd import functional, lnmod
        if case["op"] == "rows":
            return lnmod.quantize_rows(s["x"], case["code"])
        if case["op"] == "product":
            return lnmod.code_product(s["codes"], s["scales"], s["w"], s["w_scales"], s["bias"], DTYPES[case["dtype"]])
        if case["op"] == "rotary":
            ys = functional.rotary(s["q"], s["k"], s["positions"], s["table"], _axes(case), case["interleaved"])
            leaves = (s["q"], s["k"])
        else:
            ys = functional.qk_norm_rotary(s["q"], s["k"], s["wq"], s["wk"], s["positions"], s["table"], _axes(case),
                                           case["interleaved"], EPS)
            leaves = (s["q"], s["k"], s["wq"], s["wk"])
        if not case["step"]:
            return ys
        return tuple(y.detach() for y in ys) + torch.autograd.grad(ys, leaves, (s["dq"], s["dk"]))
    if case["op"] == "rows":
        q, scales = _row_codes(s["x"].float(), case["code"])
        return q.to(torch.float8_e4m3fn), scales
    return _plain_product(s) if case["op"] == "product" else _plain_attention_input(s)


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "rows":
        return {"bytes": case["M"] * (case["K"] * (e + 1) + 4), "flops": 4 * case["M"] * case["K"]}
    if case["op"] == "product":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": (M + N) * (K + 4) + M * N * e + (N * e if case["bias"] else 0), "flops": 2 * M * N * K}
    rows, T = _tokens(case)
    heads, width = case["heads"] + case["kv_heads"], sum(_axes(case))
    n = T * heads * case["head_dim"]
    passes = 5 if case["step"] and case["op"] == "qk" else 4 if case["step"] else 2     # x, y;  dy, dx;  x again for the norm
    most = max(max(f * h if len(_axes(case)) == 2 else max(f, h), w) for f, h, w in _grids(case))
    more = 4 * rows * len(_axes(case)) + most * width * 4                               # positions, cosines and sines
    if case["op"] == "qk":
        w = case["head_dim"] * (2 if case["per_head"] else heads)
        more += w * e * (2 if case["step"] else 1)
        if case["step"]:
            more += 8 * T * (heads if case["per_head"] else 2)                          # 1 / root, written and read
    return {"bytes": n * e * passes + more, "flops": n * (3 if case["op"] == "rotary" else 7) * (3 if case["step"] else 1)}


# ---- 64 bits ---------------------------------------------------------------------------------------------------------
def _to_e4m3(p):
    """Nearest e4m3 of float64 values, ties to even: 3 bits behind the leading one, steps of 2^-9 below 2^-6."""
    step = torch.exp2(torch.floor(torch.log2(p.abs().clamp_min(2.0 ** -6))) - 3.0)
    return (torch.round(p / step) * step).clamp(-448.0, 448.0)


def exact(case, seed):
    s = {k: v.detach() if isinstance(v, torch.Tensor) else v for k, v in prepare(case, seed).items()}
    if case["op"] == "rows":
        v = s["x"].double()
        scale = (v.abs().amax(-1, keepdim=True).clamp_min(SMALLEST) / LARGEST[case["code"]]).float()
        inverse = (1.0 / scale.double()).float().double()
        return _to_e4m3((v * inverse).float().double()), scale[:, 0].double()
    if case["op"] == "product":
        a = s["codes"].double() * s["scales"].double()[:, None]
        w = s["w"].double() * s["w_scales"].double()[:, None]
        y = torch.mm(a, w.t())
        return y if s["bias"] is None else y + s["bias"].double()
    axes, hd = _axes(case), case["head_dim"]
    pos = _positions(case).double()
    # pair by pair a complex factor, one column of the head's features at a time
    angles = [pos[:, a] * BASE ** (-2.0 * i / d) for a, d in enumerate(axes) for i in range(d // 2)]
    half = len(angles)
    pairs = [(2 * j, 2 * j + 1) if case["interleaved"] else (j, j + half) for j in range(half)]

    def rotate(v, sign):
        out = v.clone()
        for (a, b), t in zip(pairs, angles):
            c, z = torch.cos(t).cuda()[:, None], sign * torch.sin(t).cuda()[:, None]
            out[..., a] = v[..., a] * c - v[..., b] * z
            out[..., b] = v[..., a] * z + v[..., b] * c
        return out

    ys, grads, weights = [], [], []
    for name in ("q", "k"):
        v = s[name].double()
        n = v.shape[-2]
        if case["op"] == "qk":
            w = s["w" + name].double()
            w = w.expand(n, hd) if case["per_head"] else w.view(n, hd)
            ms = v.square().mean(-1, keepdim=True)
            root = ((ms if case["per_head"] else ms.mean(-2, keepdim=True)) + EPS).rsqrt()
            ys.append(rotate(v * root * w, 1.0))
        else:
            ys.append(rotate(v, 1.0))
        if not case["step"]:
            continue
        g = rotate(s["d" + name].double(), -1.0)
        if case["op"] == "qk":
            unit = v * root
            dw = (g * unit).reshape(-1, n, hd).sum(0)
            weights.append(dw.sum(0) if case["per_head"] else dw.reshape(-1))
            g = g * w
            dot = (g * unit).mean(-1, keepdim=True)
            g = root * (g - unit * (dot if case["per_head"] else dot.mean(-2, keepdim=True)))
        grads.append(g)
    return tuple(ys + grads + weights)
