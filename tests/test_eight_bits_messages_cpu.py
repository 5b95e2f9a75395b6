"""What the errors of the 8-bit operators say."""
import pytest
import torch

from paper_2605_17923_amd import functional, lnmod


@pytest.mark.parametrize("call", [lnmod.rmsnorm_quant_forward, functional.rms_norm_quant])
def test_an_eps_that_is_too_small_is_named(call):
    x, w = torch.zeros(5, 64, dtype=torch.bfloat16), torch.ones(64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="eps must be at least 1e-20.*got 1e-21"):
        call(x, w, eps=1e-21, group=0)
    for eps, group in ((1e-20, 0), (1e-21, 32)):                         # these reach the check of the device
        with pytest.raises(ValueError, match="GPU"):
            call(x, w, eps=eps, group=group)


def test_the_status_does_not_blame_the_width_alone():
    A = 0x1000
    st = lnmod.lnmod_rmsnorm_quant_forward(A, None, A, 4, 64, 1e-21, 0, None, None, A, A, None, A, 0, 1)
    assert st == lnmod.LNMOD_EUNSUPPORTED and "combination" in lnmod.lnmod_status_string(st)
