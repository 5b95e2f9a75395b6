"""The float64 oracle of the 8-bit codes against numbers worked out by hand, against torch's own e4m3 conversion, and (its
backward) against differences of its forward."""
import numpy as np
import pytest
import torch

from oracle import code_oracle as co


def test_int8_by_hand():
    # group of 32: amax 254 -> s = 2, r = 0.5; ties go to even
    v = np.zeros((1, 40))
    v[0, :8] = [254.0, -254.0, 1.0, 3.0, -1.0, 5.0, 2.5, 0.99]
    v[0, 32:] = [0.0, 0.0, 127.0, 0.5, 1.5, -2.5, 126.5, -126.5]           # the short last group: s = 1
    codes, s = co.encode(v, "int8", 32)
    assert s.tolist() == [[2.0, 1.0]]
    assert codes[0, :8].tolist() == [127.0, -127.0, 0.0, 2.0, 0.0, 2.0, 1.0, 0.0]
    assert codes[0, 32:].tolist() == [0.0, 0.0, 127.0, 0.0, 2.0, -2.0, 126.0, -126.0]
    assert np.array_equal(co.decode(codes, s, 32)[0, :2], [254.0, -254.0])


def test_zeros_floor_and_values_that_are_no_numbers():
    v = np.zeros((4, 32))
    v[1, 0] = 2.0 ** -120
    v[2, 5] = np.inf
    v[3, 6] = np.nan
    for code in ("int8", "e4m3"):
        codes, s = co.encode(v, code, 32)
        assert not codes.any()
        floor = np.float64(np.float32(2.0 ** -100 / co.LARGEST[code]))
        assert s[0, 0] == floor and s[1, 0] == floor and np.isnan(s[2:]).all()


def test_e4m3_is_torchs():
    p = np.concatenate([np.linspace(-460, 460, 40001), np.linspace(-0.02, 0.02, 4001), [464.0, 447.9, 2.0 ** -10, 3 * 2.0 ** -10]])
    p = p.astype(np.float32).astype(np.float64)
    p = p[np.abs(p) <= 448.0]
    want = torch.from_numpy(p).float().to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(co.to_e4m3(p), want)


@pytest.mark.parametrize("group", [32, 64, 128, 0])
@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_a_code_is_at_most_half_a_step_off(code, group):
    rng = np.random.default_rng(3)
    v = rng.normal(size=(7, 200)) * np.exp(rng.normal(size=(7, 200)) * 2)
    codes, s = co.encode(v, code, group)
    assert np.abs(codes).max() == co.LARGEST[code]
    wide = np.concatenate([np.repeat(s[:, k:k + 1], b - a, axis=1) for k, (a, b) in enumerate(co.groups_of(200, group))], axis=1)
    off = np.abs(co.decode(codes, s, group) - v)
    if code == "int8":
        assert (off <= wide * 0.5 * (1 + 1e-5)).all()          # r and s are rounded: 127 * 2^-23 on top of one half
    else:
        # half a step: 2^-4 of the value, or 2^-10 scales where the value lies below the normal codes
        assert (off <= np.maximum(np.abs(v) * 2.0 ** -4, wide * 2.0 ** -10) * (1 + 1e-6)).all()


def _slope(f, x, d, eps=1e-6):
    return (f(x + eps * d) - f(x - eps * d)) / (2 * eps)


def test_ln_backward_is_the_slope_of_its_forward():
    rng = np.random.default_rng(4)
    x, dy, dx = (rng.normal(size=(9, 24)) for _ in range(3))
    shift, scale, dsh, dsc = (rng.normal(size=(3, 24)) for _ in range(4))
    of = np.array([0, 0, 0, 0, 2, 2, 2, 2, 2])
    _, mean, rstd = co.ln_forward(x, shift, scale, of, 1e-3)
    gx, gsh, gsc = co.ln_backward(dy, x, scale, of, mean, rstd)
    loss = lambda x_, sh, sc: (co.ln_forward(x_, sh, sc, of, 1e-3)[0] * dy).sum()
    assert np.isclose((gx * dx).sum(), _slope(lambda t: loss(t, shift, scale), x, dx), rtol=1e-7)
    assert np.isclose((gsh * dsh).sum(), _slope(lambda t: loss(x, t, scale), shift, dsh), rtol=1e-7)
    assert np.isclose((gsc * dsc).sum(), _slope(lambda t: loss(x, shift, t), scale, dsc), rtol=1e-7)
    assert not gsh[1].any() and not gsc[1].any()


def test_rms_backward_is_the_slope_of_its_forward():
    rng = np.random.default_rng(5)
    h, dy, dh, d = (rng.normal(size=(6, 24)) for _ in range(4))
    w, dw = rng.normal(size=24), rng.normal(size=24)
    _, rstd = co.rms_forward(h, w, 1e-3)
    gh, gw = co.rms_backward(dy, h, w, rstd, dh)
    loss = lambda h_, w_: (co.rms_forward(h_, w_, 1e-3)[0] * dy).sum() + (h_ * dh).sum()
    assert np.isclose((gh * d).sum(), _slope(lambda t: loss(t, w), h, d), rtol=1e-7)
    assert np.isclose((gw * dw).sum(), _slope(lambda t: loss(h, t), w, dw), rtol=1e-7)
