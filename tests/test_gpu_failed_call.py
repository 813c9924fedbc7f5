"""A call that the CUDA runtime refuses says so, and leaves nothing behind for the caller's next launch."""
import ctypes

import pytest
import torch

import paper_2502_01662_b200 as pkg
from paper_2502_01662_b200 import draft
from test_draft_args import _distill, _sample, _top

pytestmark = pytest.mark.gpu

NO_DEVICE = 1 << 20


def torch_goes_on():
    assert torch.arange(1000, device="cuda").sum().item() == 499500


@pytest.mark.parametrize("make", [_sample, _top, lambda: _distill("cos_distill_loss"), lambda: _distill("cos_distill_grad"), lambda: _distill("cos_distill_step")])
def test_the_proposers_operators(make):
    torch_goes_on()
    fn, a, _ = make()
    a.device = NO_DEVICE
    assert fn(ctypes.byref(a), None) not in (0, 1, 3)
    assert b"device" in draft._library().cos_verify_last_error(None)
    torch_goes_on()


def test_a_context():
    torch_goes_on()
    with pytest.raises(pkg.CosVerifyError, match="device"):
        pkg.CosVerifier(2, pkg.COS_COMBINE_PROB_ENSEMBLE, (0.5, 0.5), 1.0, 3, 1000, 2, torch.float32, device=NO_DEVICE)
    torch_goes_on()
