"""Top logits and distillation at temperatures at which every token that is not ruled out weighs nearly the same: tokens at -inf stay ruled out, and vectors that reach over a row's ends stay out of it.

The tolerances are those of ordinary temperatures.  A factor log2(e) / T that is a multiple c of 2^-149 is off by up to 2^-149 (half of it, or all of it where it is the least), which
comes to 2^128 2^-149 ln 2 = 2^-21.5 of a term at the most, and of a sum at the most: within the 17 2^-22 that they allow for maxima that move, of which there are few here."""
import math

import pytest
import torch

import paper_2502_01662_b200 as pkg
from draft_reference import DTYPES
from test_gpu_distill import check as check_distill
from test_gpu_top import check as check_top

pytestmark = pytest.mark.gpu

HIGH = [1e30, 1e37, 1e38, 1.3e38, 1e40, 1e44, 2e45, 1e46, 1e50, 1e299]
INF = float("inf")


def rows_of(rows, V, dtype, seed):
    """Masked and whole rows, which start anywhere, among them some at the ends of what the type holds."""
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.zeros((rows, V + 3), dtype=DTYPES[dtype], device="cuda")[:, 1:V + 1]
    x.copy_(2.5 * torch.randn((rows, V), generator=g, device="cuda"))
    x[0, 7] = -INF
    x[1, ::2] = -INF
    x[2, 1:] = -INF
    x[3, 5:] = torch.finfo(x.dtype).min
    return x


@pytest.mark.parametrize("T", HIGH)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,V", [(5, 3001), (50, 40003)])
def test_top_logits(rows, V, dtype, T):
    x = rows_of(rows, V, dtype, seed=V)
    x[4] = -INF
    out = check_top(x, 40, T)
    assert bool(out["lse"][[0, 1, 2, 3]].isfinite().all()) and float(out["lse"][4]) == -INF


@pytest.mark.parametrize("T", HIGH)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,V", [(5, 3001), (40, 20001), (2, 260001)])
def test_distillation(rows, V, dtype, T):
    g = torch.Generator("cuda").manual_seed(rows)
    if rows == 2:                                      # (rows longer than a block holds, by a cluster)
        x = rows_of(4, V, dtype, seed=V)[:2]
    else:
        x = rows_of(rows, V, dtype, seed=V)
    ids = torch.randint(0, V, (rows, 2, 9), generator=g, device="cuda").int()
    ids[0, 0, 0] = 7                                   # a ruled-out token that a teacher wants
    ids[1, :, :] |= 1                                  # none of the ruled-out ones
    ids[1].clamp_(max=V - 2)
    values = torch.randn((rows, 2, 9), generator=g, device="cuda")
    lse = torch.full((rows, 2), 9.5, device="cuda")
    for l in (lse, None):
        step = check_distill(x, ids, values, l, [0.4, 0.6], T)
        assert float(step["loss"][0]) == INF and math.isfinite(float(step["loss"][1]))


def test_subnormal_numbers_flushed_on_the_host():
    """The calling thread's treatment of subnormal numbers changes nothing."""
    x = rows_of(5, 3001, "f32", seed=1)
    ids, values, rw = torch.tensor([[7, 9]] * 5, dtype=torch.int32, device="cuda"), torch.zeros((5, 2), device="cuda"), torch.ones(5, device="cuda")
    for T in (1e40, 1e50):
        want = pkg.top_logits(x, 5, T)["lse"], pkg.distill_step(x, ids, values, rw, temperature=T)["loss"]
        if not torch.set_flush_denormal(True):
            pytest.skip("not on this processor")
        try:
            got = pkg.top_logits(x, 5, T)["lse"], pkg.distill_step(x, ids, values, rw, temperature=T)["loss"]
        finally:
            torch.set_flush_denormal(False)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and bool(got[0].isfinite().all()) and float(got[1][0]) == INF
