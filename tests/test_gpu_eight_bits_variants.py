"""Every instantiation of the 8-bit row kernels at the entries of their launch-shape tables: residual or none, a scale for
the row or for a group, int8 or e4m3, codes or values, each in every width class of 512 features and every class of sizes,
where test_gpu_eight_bits_sizes.py takes one of them per entry.  References and bounds are those of that file."""
import pytest

from test_gpu_eight_bits_sizes import _memory, run_ckpt, run_rms, rows_of  # noqa: F401  (_memory is a fixture)

pytestmark = pytest.mark.gpu


def width(col, mb):
    return 512 * col - (8, 256, 64)[(col + mb) % 3]


# x on each side of 10, 50 and 200 MB (bf16) or 10 and 50 MB (fp32)
@pytest.mark.parametrize("dtype,mb", [("bf16", 8), ("bf16", 30), ("bf16", 70), ("bf16", 220), ("f32", 8), ("f32", 30), ("f32", 70)])
@pytest.mark.parametrize("col", range(1, 17))
def test_rms(col, dtype, mb):
    D = width(col, mb)
    for residual in (False, True):
        for code in ("int8", "e4m3"):
            for group in (0, (32, 64, 128)[col % 3]):
                run_rms(D, rows_of(mb, D, dtype), dtype, code, group, residual)


# x on each side of 10, 40, 50 and 200 MB (bf16) or 10 and 50 MB (fp32)
@pytest.mark.parametrize("dtype,mb", [("bf16", 8), ("bf16", 14), ("bf16", 48), ("bf16", 70), ("bf16", 220), ("f32", 8), ("f32", 14),
                                      ("f32", 60)])
@pytest.mark.parametrize("col", range(1, 17))
def test_checkpoint(col, dtype, mb):
    D = width(col, mb)
    for code in ("int8", "e4m3"):
        run_ckpt(D, rows_of(mb, D, dtype), dtype, code, (128, 32, 64)[col % 3])


@pytest.mark.parametrize("dtype,mb", [("bf16", 8), ("bf16", 14), ("bf16", 48), ("bf16", 70), ("f32", 14), ("f32", 60)])
@pytest.mark.parametrize("col", range(1, 17))
def test_checkpoint_several_segments(col, dtype, mb):
    D = width(col, mb)
    T = rows_of(mb, D, dtype)
    cuts = [0, 0, 2, T // 5, T // 5 + 1, T // 2 + 7, T // 2 + 7, T - 3, T]
    for code in ("int8", "e4m3"):
        run_ckpt(D, T, dtype, code, (64, 128, 32)[col % 3], cuts=cuts)


@pytest.mark.parametrize("dtype,mb", [("bf16", 8), ("bf16", 14), ("bf16", 210), ("f32", 8), ("f32", 14), ("f32", 210)])
@pytest.mark.parametrize("col", range(1, 17))
def test_checkpoint_per_token(col, dtype, mb):
    D = width(col, mb)
    for code in ("int8", "e4m3"):
        run_ckpt(D, rows_of(mb, D, dtype), dtype, code, (128, 64, 32)[col % 3], token=True)
