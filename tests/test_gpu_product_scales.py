"""The product of codes where the scales are far apart: y is what its formula gives wherever y itself is a float32, whatever
sum * a_scale or sum * w_scale would be.

On whole numbers of at most 8 and scales that are powers of two sum * a_scale * w_scale is exact in 64 bits.  It rounds to float32 only where
it is beyond that type's range or below 2^-126, once, and then to the result's type: bit for bit what a conversion from 64 bits
gives.  On other values: u = 2^-24; conversion, two products and bias round once each, 4 u of |y| + |bias|, and what e4m3's matrix
instruction drops (7 * 2^-13 of the largest of eight neighbouring products where y is bf16, K u of the sum of magnitudes elsewhere)."""
import pytest
import torch

from paper_2605_17923_amd import lnmod

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BOTH = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
CODES = pytest.mark.parametrize("code", ["int8", "e4m3"])
# few rows; small tiles; larger ones; 256 x 256
SIZES = pytest.mark.parametrize("size", [(3, 40, 64), (16, 257, 136), (200, 300, 264), (550, 1851, 136), (437, 17162, 512)], ids=str)
EXPONENTS = torch.tensor([-149, -140, -127, -126, -110, -109, -108, -107, -100, -60, -1, 0, 7, 60, 91, 92, 93, 100, 121, 127])


def codes_of(code, g, *shape):
    v = torch.randint(-8, 9, shape, generator=g, device="cuda", dtype=torch.int8)
    return v if code == "int8" else v.float().to(torch.float8_e4m3fn)


@BOTH
@CODES
@SIZES
def test_scales_of_any_size(size, code, dtype):
    M, N, K = size
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    a, w = codes_of(code, g, M, K), codes_of(code, g, N, K)
    at = [torch.randint(0, len(EXPONENTS), (n,), generator=g, device="cuda") for n in (M, N)]
    sa, sw = (torch.exp2(EXPONENTS.cuda().double())[i] for i in at)
    bias = torch.randn(N, generator=g, device="cuda").to(dtype)
    v = (a.double() @ w.double().t().contiguous()) * sa[:, None] * sw
    for b in (None, bias):
        y = lnmod.code_product(a, sa.float(), w, sw.float(), b, dtype)
        want = (v.float() if b is None else v.float() + b.float()).to(dtype)
        assert torch.equal(y, want), "%d of %d" % (int((y != want).sum()), y.numel())


@BOTH
@CODES
@SIZES
def test_one_sign_each_and_zero(size, code, dtype):
    """Scales below zero, and zeros, which make a row or column the bias."""
    M, N, K = size
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    a, w = codes_of(code, g, M, K), codes_of(code, g, N, K)
    sa, sw = (torch.exp2(torch.randint(-3, 4, (n,), generator=g, device="cuda").float()) for n in (M, N))
    sa[0], sa[M - 1], sw[0], sw[N - 1] = -2.0 ** 100, 0.0, -0.5, 0.0
    bias = torch.randn(N, generator=g, device="cuda").to(dtype)
    v = (a.double() @ w.double().t().contiguous()) * sa.double()[:, None] * sw.double()
    assert torch.equal(lnmod.code_product(a, sa, w, sw, bias, dtype), (v.float() + bias.float()).to(dtype))


@BOTH
@CODES
@SIZES
@pytest.mark.parametrize("largest", [1e-30, 1e33, 1e35, None], ids=str)
def test_rows_of_large_values_by_ordinary_weights(largest, size, code, dtype):
    """What quantize_rows makes of rows up to the type's largest value, by weights of about 0.02, and of large weights by ordinary
    rows."""
    M, N, K = size
    g = torch.Generator(device="cuda").manual_seed(M + 2 * N + K)
    x = torch.randn(M, K, generator=g, device="cuda")
    x = x / x.abs().amax(-1, keepdim=True)
    x[::2] *= torch.finfo(dtype).max if largest is None else largest
    w = torch.randn(N, K, generator=g, device="cuda") * 0.02 / K
    w[::3] *= 1e-3
    (ca, sa), (cw, sw) = lnmod.quantize_rows(x.to(dtype), code), lnmod.quantize_rows(w.to(dtype), code)
    for a, s, b, t in ((ca, sa, cw, sw), (cw[:M], sw[:M], ca[:, :].repeat(-(-N // M), 1)[:N], sa.repeat(-(-N // M))[:N])):
        ad, bd, scale = a.double(), b.double(), s.double()[:, None] * t.double()
        v = (ad @ bd.t().contiguous()) * scale
        assert float(v.abs().amax()) < 1e38
        slack = 4 * U * v.abs()
        if code == "e4m3":
            slack = slack + K * U * (ad.abs() @ bd.abs().t().contiguous()) * scale
            if dtype == torch.bfloat16:
                for k in range(0, K, 8):                             # at most the product of the two largest of the eight
                    slack = slack + 7 * 2.0 ** -13 * ad[:, None, k:k + 8].abs().amax(-1) * bd[:, k:k + 8].abs().amax(-1) * scale
        y = lnmod.code_product(a.contiguous(), s.contiguous(), b.contiguous(), t.contiguous(), None, dtype)
        err = (y.double() - v).abs()
        # below 2^-126 the type's steps are 2^-126 eps whatever the value, and float32's, which comes first, are 2^-149
        tol = torch.finfo(dtype).eps / 2 * (v.abs() + 2.0 ** -126) + slack + 2.0 ** -149
        assert y.shape == v.shape and bool((err <= tol).all()), int((~(err <= tol)).sum())
