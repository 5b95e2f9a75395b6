"""Which kernels the sizes of the product's GPU tests take, by the library's own rule: each of the ten is reached, to either type, and
each size of test_gpu_product_large.py takes the kernel that stands beside it, with its outputs where that file says.  So a change of
the rule cannot quietly leave a kernel untested.  Needs only hipcc's host compiler."""
import os
import shutil

import pytest

import product_plan
import test_gpu_code_product as first
import test_gpu_product_edges as edges
import test_gpu_product_large as large
from paper_2605_17923_amd import build

FORMS = [(code, dtype) for code in ("int8", "e4m3") for dtype in ("bf16", "f32")]


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    if shutil.which(build._hipcc()) is None and not os.path.exists(build._hipcc()):
        pytest.skip("hipcc not found")
    exe = product_plan.program(tmp_path_factory.mktemp("plan"))
    return lambda problems: product_plan.plans(problems, exe)


@pytest.mark.parametrize("form", FORMS, ids=str)
def test_every_kernel_has_a_size(form, plans):
    halves = form == ("e4m3", "f32")
    reached = {k for k, _ in plans([s + form for s in edges.SIZES])}
    assert reached == set(range(9 if halves else 10))
    reached = {k for k, _ in plans([s + form for s in first.SIZES])}
    assert reached >= {0, 1, 2, 3, 4}


@pytest.mark.parametrize("form", FORMS, ids=str)
def test_the_large_sizes_take_the_kernels_beside_them(form, plans):
    halves = form == ("e4m3", "f32")
    for table in (large.PAST, large.LONG, large.LONGEST, large.FAR):
        got = plans([s + form for s in table])
        assert [k for k, _ in got] == [pair[halves] for pair in table.values()]
        if table is large.PAST:
            kept = [s for s, (_, keep) in zip(table, got) if keep]
            assert kept == (large.KEPT_IN_BF16 if form[1] == "bf16" else [])
