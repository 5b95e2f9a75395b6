"""The workspace queries of the 8-bit backwards on one sample: a workspace that holds the longest batch serves every shorter one."""
import pytest

from paper_2605_17923_amd import lnmod

WIDTHS = [8, 200, 512, 520, 1000, 1024, 1536, 2048, 2560, 2600, 3584, 4096, 5120, 6144, 8192]
# every row count around the lines where a block gets another wave, then ever longer ones
ROWS = sorted(set(list(range(0, 6200)) + [k << s for s in range(8, 30) for k in (3, 4, 5, 7)]
                  + [(n << 20) // (16 * D) + d for n in (10, 40, 48, 50, 52) for D in WIDTHS for d in (-1, 0, 1)]))


@pytest.mark.parametrize("D", WIDTHS)
def test_the_queries_of_one_sample_never_fall(D):
    for query in (lambda n: lnmod.lnmod_backward_ckpt_workspace_bytes(1, n, D),
                  lambda n: lnmod.lnmod_rmsnorm_quant_backward_workspace_bytes(n, D)):
        sizes = [query(n) for n in ROWS if 0 <= n < 1 << 31]
        assert all(a <= b for a, b in zip(sizes, sizes[1:])), D
        assert sizes[0] == 0 and sizes[1] > 0


def test_a_workspace_of_the_longer_batch_is_taken_for_the_shorter_one():
    # 257 to 511 rows of one wave each: two rows to a block, fewer blocks than 256 rows have
    A = 0x1000
    for D, long, short in ((512, 300, 256), (1536, 513, 512), (2560, 700, 511)):
        ws = lnmod.lnmod_rmsnorm_quant_backward_workspace_bytes(long, D)
        call = lambda n, rstd: lnmod.lnmod_rmsnorm_quant_backward(A, None, A, A, n, D, None, rstd, A, A, A + 4, ws, 0, 0)
        assert call(short, None) == lnmod.LNMOD_EINVAL                   # refused for the pointer ...
        assert call(short, A) == lnmod.LNMOD_EALIGN                      # ... or the address, not for the size
        ws = lnmod.lnmod_backward_ckpt_workspace_bytes(1, long, D)
        assert lnmod.lnmod_backward_ckpt(A, A, A, A, None, 1, short, D, 32, None, A, A, A, A, A, A + 4, ws, 0, 0, 0,
                                         0) == lnmod.LNMOD_EALIGN
