"""The product of codes where it is large: sizes of the 256 x 256 kernel and outputs that go past the caches, with codes of the full
range, long sums and operands beyond 4 GiB.  Which kernel each size takes stands beside it; test_product_plan_cpu.py holds the
library's rule to that.

On whole numbers of at most 8 with scales that are powers of two everything but the last rounding is exact (sums below 2^24), so the
outputs are float32's bit for bit.  On codes of the full range: u = 2^-24; int8 sums are exact, their conversion, the two products and
the bias round once each, 4 u of |y| + |bias|; e4m3 sums to float32 are off by K u of the sum of magnitudes in any order; e4m3 sums to
bf16 besides by less than 7 * 2^-13 of the sum, over eight neighbouring features each, of their largest product."""
import pytest
import torch

from paper_2605_17923_amd import lnmod

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
KIND = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
BOTH = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
CODES = pytest.mark.parametrize("code", ["int8", "e4m3"])
TWO, FIVE, SIX, SEVEN, EIGHT, LARGE = 2, 5, 6, 7, 8, 9

# (M, N, K): the kernel, the one for e4m3 codes to float32.  Outputs past the caches in either type, but for those of 222 933 x 128 and
# 1217 x 26 304 in bf16.
PAST = {(9, 4283456, 72): (TWO, TWO),
        (583795, 64, 3704): (FIVE, FIVE),
        (222933, 128, 8000): (SIX, SEVEN),
        (324331, 128, 2280): (SEVEN, SEVEN),
        (8200, 4416, 136): (SEVEN, EIGHT),
        (1217, 26304, 16): (SEVEN, EIGHT),
        (4609, 8192, 264): (EIGHT, EIGHT),
        (16500, 4224, 384): (LARGE, EIGHT),                  # an odd number of steps, tiles that end in M and in N
        (8200, 8256, 264): (LARGE, EIGHT),                   # a tail in K
        (3000, 24640, 392): (LARGE, EIGHT),                  # four and five tiles a block
        (2305, 16384, 5128): (LARGE, EIGHT)}
KEPT_IN_BF16 = [(222933, 128, 8000), (1217, 26304, 16)]
# outputs that stay in the caches, or do not, as it comes
LONG = {(437, 17162, 5128): (LARGE, SEVEN), (5121, 7001, 5120): (LARGE, SEVEN), (19001, 2368, 5120): (LARGE, EIGHT)}
LONGEST = {(4097, 8256, 131064): (LARGE, SEVEN)}
FAR = {(33000, 4352, 131064): (LARGE, EIGHT)}                # a: 4.3e9 bytes


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def whole(code, g, rows, K):
    v = torch.empty(rows, K, dtype=KIND[code], device="cuda")
    for i in range(0, rows, 8192):
        part = torch.randint(-8, 9, v[i:i + 8192].shape, generator=g, device="cuda", dtype=torch.int8)
        v[i:i + 8192] = part if code == "int8" else part.float().to(KIND[code])
    return v


def full(code, g, rows, K):
    if code == "int8":
        return torch.randint(-128, 128, (rows, K), generator=g, device="cuda", dtype=torch.int8)
    v = torch.randn(rows, K, generator=g, device="cuda") * 40
    v *= torch.where(torch.rand(rows, K, generator=g, device="cuda") < 1e-3, 10.0, 1.0)
    return v.clamp(-448, 448).to(KIND[code])


def fenced(a, sa, w, sw, b, dtype):
    """The product, written between two stretches of memory that have to stay as they are."""
    M, K, N, fence = a.shape[0], a.shape[1], w.shape[0], 4096
    y = torch.full((2 * fence + M * N,), 7.0, dtype=dtype, device="cuda")
    st = lnmod.lnmod_code_product(a, sa, w, sw, b, M, N, K, torch.cuda.current_stream().cuda_stream, y[fence:].data_ptr(),
                                  lnmod.LNMOD_BF16 if dtype == torch.bfloat16 else lnmod.LNMOD_F32,
                                  lnmod.LNMOD_INT8 if a.dtype == torch.int8 else lnmod.LNMOD_E4M3)
    assert st == lnmod.LNMOD_OK
    assert bool((y[:fence] == 7).all()) and bool((y[fence + M * N:] == 7).all())
    return y[fence:fence + M * N].view(M, N)


@BOTH
@CODES
@pytest.mark.parametrize("size", list(PAST) + list(LONG), ids=str)
def test_whole_numbers(size, code, dtype):
    M, N, K = size
    g = generator(M + N + K)
    a, w = whole(code, g, M, K), whole(code, g, N, K)
    sa, sw = (torch.exp2(torch.randint(-3, 4, (n,), generator=g, device="cuda").float()) for n in (M, N))
    bias = torch.randn(N, generator=g, device="cuda").to(dtype)
    v = (a.float() @ w.float().t().contiguous()) * sa[:, None] * sw
    for b in (None, bias):
        y = fenced(a, sa, w, sw, b, dtype)
        assert torch.equal(y, (v if b is None else v + b.float()).to(dtype))
        assert torch.equal(lnmod.code_product(a, sa, w, sw, b, dtype), y)          # the same bits again


@BOTH
@CODES
@pytest.mark.parametrize("size", [(4609, 8192, 264), (8200, 8256, 264), (2305, 16384, 5128)] + list(LONG), ids=str)
def test_codes_of_the_full_range(size, code, dtype):
    M, N, K = size
    g = generator(M + N + K + 1)
    a, w = full(code, g, M, K), full(code, g, N, K)
    sa, sw = (torch.rand(n, generator=g, device="cuda") * 0.01 + 1e-3 for n in (M, N))
    b = torch.randn(N, generator=g, device="cuda").to(dtype)
    y = lnmod.code_product(a, sa, w, sw, b, dtype)

    def sampled(n):
        picks = [0, 1, 127, 128, 255, 256, n // 2, n - 1] + torch.randint(0, n, (16,), generator=g, device="cuda").tolist()
        return torch.tensor(sorted({p for p in picks if p < n}), device="cuda")

    for rows, cols in ((sampled(M), slice(0, N)), (slice(0, M), sampled(N))):
        ad, wd = a[rows].double(), w[cols].double()
        scale = sa[rows].double()[:, None] * sw[cols].double()
        v = torch.mm(ad, wd.t().contiguous()) * scale
        want = v + b[cols].double()
        slack = 4 * U * (v.abs() + b[cols].double().abs())
        if code == "e4m3":
            slack = slack + K * U * torch.mm(ad.abs(), wd.abs().t().contiguous()) * scale
            if dtype == torch.bfloat16:
                most = torch.zeros_like(v)
                for k in range(0, K, 8):
                    eight = torch.zeros_like(v)
                    for j in range(k, k + 8):
                        eight = torch.maximum(eight, ad[:, j].abs()[:, None] * wd[:, j].abs())
                    most += eight
                slack = slack + 7 * 2.0 ** -13 * most * scale
        err = (y[rows][:, cols].double() - want).abs()
        tol = torch.finfo(dtype).eps / 2 * want.abs() + slack
        assert bool((err <= tol).all()), "%d values off, worst %.3g of the bound" % (int((err > tol).sum()), float((err / tol).max()))


@BOTH
@pytest.mark.parametrize("size", list(LONGEST), ids=str)
def test_the_longest_sum_of_the_largest_codes(size, dtype):
    """131 064 products of 128 x 128 and of -128 x 127: exact in 32 bits, then one rounding to float32 and one to the result's type."""
    M, N, K = size
    a, w = (torch.full((n, K), -128, dtype=torch.int8, device="cuda") for n in (M, N))
    w[1::2] = 127
    y = fenced(a, torch.ones(M, device="cuda"), w, torch.ones(N, device="cuda"), None, dtype)
    want = torch.where(torch.arange(N, device="cuda") % 2 == 0, float(K * 128 * 128), float(-K * 128 * 127)).to(dtype)
    assert torch.equal(y, want.expand(M, N))


@BOTH
@CODES
@pytest.mark.parametrize("size", list(FAR), ids=str)
def test_operands_beyond_four_gigabytes(size, code, dtype):
    M, N, K = size
    g = generator(M)
    a, w = whole(code, g, M, K), whole(code, g, N, K)
    sa, sw = (torch.exp2(torch.randint(-3, 4, (n,), generator=g, device="cuda").float()) for n in (M, N))
    y = lnmod.code_product(a, sa, w, sw, None, dtype)
    for m in (slice(0, 130), slice(M // 2 - 70, M // 2 + 70), slice(M - 200, M)):
        v = (a[m].float() @ w.float().t().contiguous()) * sa[m][:, None] * sw
        assert torch.equal(y[m], v.to(dtype))
