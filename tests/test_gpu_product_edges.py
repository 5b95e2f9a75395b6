"""Codes with one scale for a row, and their product: every kernel that the sizes can pick, values that are no numbers, extremes,
addresses, offsets beyond 32 bits, what lies around the outputs.

On whole numbers of at most 8 the sums stay below 2^24 and the scales are powers of two, so the products are exact in float32 and
only the bias and the result's type round, once each: the outputs are what float32 gives, bit for bit."""
import pytest
import torch

from paper_2605_17923_amd import lnmod

pytestmark = pytest.mark.gpu
KIND = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
BOTH = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
CODES = pytest.mark.parametrize("code", ["int8", "e4m3"])


def whole(code, g, *shape):
    v = torch.randint(-8, 9, shape, generator=g, device="cuda", dtype=torch.int8)
    return v if code == "int8" else v.float().to(KIND[code])


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def operands(code, dtype, M, N, K, bias, seed=0):
    g = generator(seed + M + 3 * N + 7 * K)
    sa, sw = (torch.exp2(torch.randint(-3, 4, (n,), generator=g, device="cuda").float()) for n in (M, N))
    b = torch.randn(N, generator=g, device="cuda").to(dtype) if bias else None
    return whole(code, g, M, K), sa, whole(code, g, N, K), sw, b


def plain(a, sa, w, sw, b, dtype):
    v = (a.float() @ w.float().t().contiguous()) * sa[:, None] * sw
    return (v if b is None else v + b.float()).to(dtype)


# Each line is one kernel's at most of these lengths: few rows; 32 x 32 and 32 x 64 outputs; 64 x 64; 96 x 64; 128 x 64; 128 x 128
# by eight waves and by four; 128 x 256; 256 x 256, with an odd and an even number of steps, a tail, one block or several for a CU.
SIZES = [(1, 5120, 5120), (5, 999, 4104), (16, 4096, 2048), (1, 7, 13824), (11, 19578, 288),
         (40, 1500, 1024), (7, 8200, 1536), (1, 15360, 5120), (200, 1433, 520), (300, 2048, 640),
         (550, 1851, 136), (1560, 654, 136), (438, 2306, 16), (3694, 396, 136), (928, 1630, 136), (413, 3368, 152), (2140, 736, 136),
         (420, 2366, 16), (3551, 284, 16), (513, 2942, 16), (3034, 2612, 16), (2403, 3417, 16), (2305, 1900, 256), (4100, 4104, 1416),
         (392, 16471, 136), (18213, 405, 200), (387, 16743, 256), (774, 9573, 264), (16415, 409, 384), (437, 17162, 512),
         (402, 17030, 520), (421, 17666, 640), (17737, 407, 1000), (396, 17423, 1416), (8200, 8200, 136), (9001, 8208, 264),
         (5121, 7001, 2056)]


@BOTH
@CODES
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_every_kernel_on_whole_numbers(size, code, dtype):
    for bias in (False, True):
        a = operands(code, dtype, *size, bias)
        assert torch.equal(lnmod.code_product(*a, dtype), plain(*a, dtype))


@BOTH
@pytest.mark.parametrize("size", [(1, 33), (16, 300), (100, 100), (600, 515), (2049, 2300)], ids=str)
def test_the_longest_sum_of_the_largest_codes(size, dtype):
    """131 064 products of 128 x 128: one step of 32 bits less would not hold them.  The sum is exact, then one rounding to float32
    and one to the result's type."""
    K = (1 << 17) - 8
    a, w = (torch.full((n, K), -128, dtype=torch.int8, device="cuda") for n in size)
    w[1::2] = 127
    y = lnmod.code_product(a, torch.ones(size[0], device="cuda"), w, torch.ones(size[1], device="cuda"), None, dtype)
    want = torch.where(torch.arange(size[1], device="cuda") % 2 == 0, float(K * 128 * 128), float(-K * 128 * 127)).to(dtype)
    assert torch.equal(y, want.expand(size))


@BOTH
@CODES
@pytest.mark.parametrize("size", [(3, 40, 64), (16, 257, 136), (200, 300, 264), (550, 1851, 136), (2305, 1900, 256), (437, 17162, 512)],
                         ids=str)
def test_values_that_are_no_numbers_stay_in_their_row_and_column(size, code, dtype):
    M, N, K = size
    a, sa, w, sw, b = operands(code, dtype, M, N, K, True)
    want = plain(a, sa, w, sw, b, dtype)
    sa[M // 2], sw[N // 3] = float("nan"), float("nan")
    rows, cols = [M // 2], [N // 3]
    b[N - 1] = float("nan")
    cols.append(N - 1)
    if code == "e4m3":
        a.view(torch.uint8)[M - 1, K - 1] = 0x7f                     # a code that is NaN
        w.view(torch.uint8)[0, K // 2] = 0xff
        rows.append(M - 1)
        cols.append(0)
    y = lnmod.code_product(a, sa, w, sw, b, dtype)
    nan = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    nan[rows] = True
    nan[:, cols] = True
    assert bool(y[nan].isnan().all()) and torch.equal(y[~nan], want[~nan])
    sa[M // 2], sw[N // 3] = float("inf"), 1.0
    y = lnmod.code_product(a, sa, w, sw, None, dtype)[M // 2]
    assert not bool(y.isfinite().any())


@BOTH
@CODES
@pytest.mark.parametrize("size", [(3, 1001, 520), (130, 1001, 264), (700, 2000, 72), (2305, 1900, 256), (402, 17030, 520)], ids=str)
def test_scales_and_bias_at_any_address_and_nothing_written_beside_y(size, code, dtype):
    M, N, K = size
    a, sa, w, sw, b = operands(code, dtype, M, N, K, True)
    want = plain(a, sa, w, sw, b, dtype)

    def moved(t):
        return torch.cat([t.new_full((3,), float("nan")), t])[3:]

    fence = 4096
    y = torch.full((2 * fence + M * N,), 7.0, dtype=dtype, device="cuda")
    at = y[fence:fence + M * N]
    moves = moved(sa), moved(sw), moved(b)
    st = lnmod.lnmod_code_product(a.data_ptr(), moves[0].data_ptr(), w.data_ptr(), moves[1].data_ptr(), moves[2].data_ptr(), M, N, K,
                                  torch.cuda.current_stream().cuda_stream, at.data_ptr(),
                                  lnmod.LNMOD_BF16 if dtype == torch.bfloat16 else lnmod.LNMOD_F32, 0 if code == "int8" else 1)
    assert st == lnmod.LNMOD_OK
    assert torch.equal(at.view(M, N), want) and bool((y[:fence] == 7).all()) and bool((y[fence + M * N:] == 7).all())


@CODES
def test_shapes(code):
    g = generator(3)
    w, sw = whole(code, g, 24, 72), torch.rand(24, generator=g, device="cuda")
    for lead in ((), (5,), (2, 3), (2, 0, 3), (0,)):
        a, sa = whole(code, g, *lead, 72), torch.ones(lead, device="cuda")
        for dtype in (torch.bfloat16, torch.float32):
            y = lnmod.code_product(a, sa, w, sw, None, dtype)
            assert y.shape == lead + (24,) and y.dtype == dtype
            if a.numel():
                flat = lnmod.code_product(a.view(-1, 72), sa.view(-1), w, sw, None, dtype)
                assert torch.equal(y.reshape(-1, 24), flat)
    assert lnmod.code_product(a, sa, w[:0], sw[:0], None, torch.float32).shape == (0, 0)
    for lead in ((0,), (2, 0)):
        codes, scales = lnmod.quantize_rows(torch.empty(*lead, 64, device="cuda"), code)
        assert codes.shape == lead + (64,) and scales.shape == lead and codes.dtype == KIND[code]


@CODES
def test_outputs_and_codes_beyond_four_gigabytes(code):
    """The last rows and columns are what they are by themselves."""
    for M, N, K in ((70001, 32776, 8), (40009, 16, 131064), (9, 40008, 131064)):
        g = generator(M)
        a, w = whole(code, g, M, K), whole(code, g, N, K)
        sa, sw = torch.rand(M, generator=g, device="cuda"), torch.rand(N, generator=g, device="cuda")
        y = lnmod.code_product(a, sa, w, sw, None, torch.bfloat16)
        for m in (slice(0, 3), slice(M // 2, M // 2 + 2), slice(M - 5, M)):
            n = slice(N - min(N, 1000) // 8 * 8, N)
            v = (a[m].float().cpu() @ w[n].float().cpu().t()).cuda() * sa[m][:, None] * sw[n]
            assert torch.equal(y[m, n], v.to(torch.bfloat16))
        del a, w, y


@BOTH
@CODES
def test_rows_beyond_four_gigabytes(code, dtype):
    N, D = (70001, 32776) if dtype == torch.bfloat16 else (35001, 32776)
    x = torch.empty(N, D, dtype=dtype, device="cuda")
    x.copy_(torch.randn(1, D, device="cuda", generator=generator(1)).to(dtype))
    last = torch.randn(64, D, device="cuda", generator=generator(2)).to(dtype)
    x[-64:] = last
    codes, scales = lnmod.quantize_rows(x, code)
    for part, want in ((slice(N - 64, N), last), (slice(0, 2), x[:2].clone()), (slice(N // 2, N // 2 + 1), x[:1].clone())):
        c, s = lnmod.quantize_rows(want, code)
        assert torch.equal(codes[part].view(torch.uint8), c.view(torch.uint8)) and torch.equal(scales[part], s)


@BOTH
@CODES
@pytest.mark.parametrize("D", [8, 24, 512, 1536, 5120, 13824, 32776])
def test_rows_that_are_no_numbers(D, code, dtype):
    """A row with an infinity or NaN has a scale of NaN and codes of zero; zeros have codes of zero and a scale that is a number;
    the rows beside them do not change."""
    x = torch.randn(37, D, device="cuda", generator=generator(D)).to(dtype)
    clean, cs = lnmod.quantize_rows(x, code)
    bad = {0: float("nan"), 9: float("inf"), 10: float("-inf"), 36: float("nan")}
    y = x.clone()
    for k, (row, v) in enumerate(bad.items()):
        y[row, (k * 7919) % D] = v
    y[17] = 0.0
    y[18] = torch.finfo(dtype).tiny
    y[19] = torch.finfo(dtype).max
    codes, scales = lnmod.quantize_rows(y, code)
    for row in range(37):
        c, s = codes[row].float(), scales[row]
        if row in bad:
            assert bool(s.isnan()) and bool((c == 0).all())
        elif row == 17:
            assert bool(s.isfinite()) and bool((c == 0).all())
        elif row in (18, 19):
            assert bool(s.isfinite()) and bool(s > 0)
        else:
            assert torch.equal(c, clean[row].float()) and torch.equal(s, cs[row])
    back = lnmod.dequantize(codes, scales, torch.float32, 0)
    assert bool(back[list(bad)].isnan().all()) and bool((back[17] == 0).all())
    prod = lnmod.code_product(codes, scales, clean[:5], cs[:5], None, torch.float32)
    assert bool(prod[list(bad)].isnan().all()) and bool(prod[[1, 2, 17, 35]].isfinite().all())


@BOTH
@CODES
@pytest.mark.parametrize("shape", [(1, 8), (5, 72), (130, 520), (9, 5128), (3, 32776)], ids=str)
def test_nothing_is_written_beside_the_codes(shape, code, dtype):
    x = torch.randn(*shape, device="cuda", generator=generator(4)).to(dtype)
    want, ws = lnmod.quantize_rows(x, code)
    n, fence = x.numel(), 1024
    codes = torch.full((n + 2 * fence,), 0x33, dtype=torch.uint8, device="cuda")
    scales = torch.full((shape[0] + 2 * fence + 1,), 7.0, device="cuda")
    at = scales[fence + 1:fence + 1 + shape[0]]                          # scales at an odd element
    st = lnmod.lnmod_quantize_rows(x.data_ptr(), *shape, torch.cuda.current_stream().cuda_stream, codes[fence:].data_ptr(), at.data_ptr(),
                                   lnmod.LNMOD_BF16 if dtype == torch.bfloat16 else lnmod.LNMOD_F32, 0 if code == "int8" else 1)
    assert st == lnmod.LNMOD_OK
    assert torch.equal(codes[fence:fence + n], want.view(torch.uint8).flatten()) and torch.equal(at, ws)
    assert bool((codes[:fence] == 0x33).all()) and bool((codes[fence + n:] == 0x33).all())
    assert bool((scales[:fence + 1] == 7).all()) and bool((scales[fence + 1 + shape[0]:] == 7).all())
