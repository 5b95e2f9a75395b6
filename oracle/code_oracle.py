"""Independent float64 oracle of the 8-bit codes (numpy, no code shared with the library): the definition that
include/lnmod.h states, group by group.

    amax = max |v|     s = fp32(max(amax, 2^-100) / Q)     r = fp32(1 / s)     Q = 127 (int8), 448 (e4m3)
    int8: rne(v*r), one rounding     e4m3: nearest e4m3 of fp32(v*r), ties to even
    a group with an infinity or a NaN: s = NaN, codes 0
"""
import numpy as np

LARGEST = {"int8": 127.0, "e4m3": 448.0}


def _f32(a):
    return np.asarray(a, dtype=np.float64).astype(np.float32).astype(np.float64)


def to_e4m3(p):
    """Nearest e4m3 value (three bits behind the leading one, steps of 2^-9 below 2^-6, largest 448), ties to even."""
    a = np.abs(p)
    _, e = np.frexp(np.maximum(a, 2.0 ** -6))                  # a = m 2^e, m in [1/2, 1)
    step = np.ldexp(1.0, e - 4)
    return np.copysign(np.minimum(np.round(a / step) * step, 448.0), p)


def groups_of(D, group):
    return [(at, min(at + group, D)) for at in range(0, D, group)] if group else [(0, D)]


def quotients(v, code, group, scales=None):
    """v [N, D] (float64, finite) -> (scales [N, groups], v*r in float64 without its rounding)."""
    q = np.empty_like(v)
    out = []
    for k, (a, b) in enumerate(groups_of(v.shape[-1], group)):
        s = _f32(np.maximum(np.abs(v[:, a:b]).max(axis=1), 2.0 ** -100) / LARGEST[code]) if scales is None else scales[:, k]
        q[:, a:b] = v[:, a:b] * _f32(1.0 / s)[:, None]
        out.append(s)
    return np.stack(out, axis=1), q


def round_code(q, code):
    return np.round(q) + 0.0 if code == "int8" else to_e4m3(_f32(q))      # a whole number has no negative zero


def encode(v, code, group):
    """v [N, D] -> (values of the codes, scales [N, groups]), float64."""
    v = np.asarray(v, dtype=np.float64)
    bad = np.stack([~np.isfinite(v[:, a:b]).all(axis=1) for a, b in groups_of(v.shape[-1], group)], axis=1)
    wide = np.zeros(v.shape, dtype=bool)
    for k, (a, b) in enumerate(groups_of(v.shape[-1], group)):
        wide[:, a:b] = bad[:, k:k + 1]
    scales, q = quotients(np.where(wide, 0.0, v), code, group)
    codes = np.where(wide, 0.0, round_code(q, code))
    return codes, np.where(bad, np.nan, scales)


def decode(codes, scales, group):
    out = np.empty(codes.shape, dtype=np.float64)
    for k, (a, b) in enumerate(groups_of(codes.shape[-1], group)):
        out[:, a:b] = codes[:, a:b] * scales[:, k:k + 1]
    return out


def ln_forward(x, shift, scale, of, eps):
    """x [T, D], shift, scale [n, D] (float64), of [T]: the modulation row of each token -> y, mean, rstd."""
    mean = x.mean(axis=1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(axis=1) + eps)
    return (x - mean[:, None]) * rstd[:, None] * (1.0 + scale[of]) + shift[of], mean, rstd


def ln_backward(dy, x, scale, of, mean, rstd):
    """From the values x that the backward reads and given statistics -> dx, dshift, dscale."""
    xhat = (x - mean[:, None]) * rstd[:, None]
    g = dy * (1.0 + scale[of])
    dx = rstd[:, None] * (g - g.mean(axis=1, keepdims=True) - xhat * (g * xhat).mean(axis=1, keepdims=True))
    dshift, dscale = np.zeros(scale.shape), np.zeros(scale.shape)
    np.add.at(dshift, of, dy)
    np.add.at(dscale, of, dy * xhat)
    return dx, dshift, dscale


def rms_forward(h, w, eps):
    rstd = 1.0 / np.sqrt((h ** 2).mean(axis=1) + eps)
    return h * rstd[:, None] * w, rstd


def rms_backward(dy, h, w, rstd, dh=None):
    hhat = h * rstd[:, None]
    g = dy * w
    dx = rstd[:, None] * (g - hhat * (g * hhat).mean(axis=1, keepdims=True))
    return dx if dh is None else dx + dh, (dy * hhat).sum(axis=0)
