"""cos_top_logits against sorting in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2502_01662_b200 as pkg
from draft_reference import DTYPES, lse_error, top_of

pytestmark = pytest.mark.gpu


def check(x, k, T):
    out = pkg.top_logits(x, k, T)
    rows, V = x.shape
    assert out["values"].shape == out["ids"].shape == (rows, k) and out["lse"].shape == (rows,)
    host = x.double().cpu().numpy()
    got = {n: v.double().cpu().numpy() for n, v in out.items()}
    for r in range(rows):
        v, ids, lse = top_of(host[r], k, float(T))
        assert np.array_equal(got["ids"][r], ids), (r, got["ids"][r], ids)
        assert np.array_equal(got["values"][r], v)
        if not math.isfinite(lse):
            assert got["lse"][r] == lse or (math.isnan(lse) and math.isnan(got["lse"][r]))
        else:
            assert abs(got["lse"][r] - lse) <= lse_error(V) + abs(lse) * 2.0 ** -24, (got["lse"][r], lse)
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,V,ks", [(1, 1, (1,)), (3, 7, (1, 7)), (2, 64, (5, 64)), (5, 1000, (1, 64, 1000)), (4, 20001, (64, 1024)), (1, 151936, (64, 512)), (160, 4099, (32,)), (700, 300, (17,))])
def test_sizes(rows, V, ks, dtype):
    g = torch.Generator("cuda").manual_seed(V)
    x = (2.5 * torch.randn((rows, V), generator=g, device="cuda")).to(DTYPES[dtype])
    for k in ks:
        check(x, k, 1.0)
        check(x, k, 2.5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(1, 0), (3, 5), (8, 8)])
def test_rows_that_start_anywhere(dtype, pad, shift):
    g = torch.Generator("cuda").manual_seed(pad)
    buf = torch.zeros(6 * (5003 + pad) + shift, dtype=DTYPES[dtype], device="cuda")
    x = buf[shift:].view(6, 5003 + pad)[:, :5003]
    x.copy_(2.0 * torch.randn((6, 5003), generator=g, device="cuda"))
    buf.view(-1)[:shift] = 99.0
    x.as_strided((6, pad), (5003 + pad, 1), shift + 5003).fill_(99.0)      # (what is not the row's)
    check(x, 50, 1.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_ties_and_masks(dtype):
    V = 40001
    g = torch.Generator("cuda").manual_seed(3)
    x = torch.randint(0, 3, (9, V), generator=g, device="cuda").to(DTYPES[dtype])
    x[1] = 0.5                                     # all alike
    x[2] = -float("inf")
    x[3, 10:] = -float("inf")                      # fewer than k
    x[4, 5] = float("nan")
    x[5, 7] = float("inf")
    x[6] = torch.finfo(x.dtype).min
    x[7, 1:] = torch.finfo(x.dtype).min
    x[8] = torch.linspace(-1, 1, V, device="cuda").to(x.dtype) * 0.01     # all in a few bins
    for k in (1, 64, 1024):
        check(x, k, 1.0)


def test_equal_zeros():
    x = torch.zeros((1, 100), device="cuda")
    x[0, ::2] = -0.0
    assert pkg.top_logits(x, 5)["ids"].tolist() == [[0, 1, 2, 3, 4]]


@pytest.mark.parametrize("T", [1e-30, 1e-3, 1e4])
def test_temperatures(T):
    g = torch.Generator("cuda").manual_seed(3)
    check(2.0 * torch.randn((3, 5000), generator=g, device="cuda"), 40, T)


def test_rows_longer_than_shared_memory():
    g = torch.Generator("cuda").manual_seed(3)
    check(torch.randn((2, 1_200_007), generator=g, device="cuda"), 300, 1.0)


def test_offsets_past_32_bits():
    V, stride = 1000, (1 << 31) + 24
    buf = torch.empty(2 * stride + V, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((3, V), (stride, 1))
    x.copy_(torch.randn((3, V), generator=torch.Generator("cuda").manual_seed(1), device="cuda"))
    check(x, 60, 1.0)


def test_streams_and_graphs():
    g = torch.Generator("cuda").manual_seed(3)
    x = torch.randn((6, 30000), generator=g, device="cuda")
    want = check(x, 64, 1.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = pkg.top_logits(x, 64, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(other[n], want[n]) for n in want)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = pkg.top_logits(x, 64)
    x.copy_(torch.randn((6, 30000), generator=g, device="cuda"))
    for _ in range(3):
        graph.replay()
    fresh = check(x, 64, 1.0)
    assert all(torch.equal(out[n], fresh[n]) for n in out)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_many_rows(dtype):
    """Rows enough for a block each: masks, ties and rows that are not finite among ordinary ones, unaligned rows."""
    V, rows = 20001, 310
    g = torch.Generator("cuda").manual_seed(5)
    x = (2.5 * torch.randn((rows, V), generator=g, device="cuda")).to(DTYPES[dtype])
    x[1] = 0.5
    x[2] = -float("inf")
    x[3, 10:] = -float("inf")
    x[4, 5] = float("nan")
    x[5, 7] = float("inf")
    x[6] = torch.finfo(x.dtype).min
    x[7, 1:] = torch.finfo(x.dtype).min
    x[8] = torch.randint(0, 3, (V,), generator=g, device="cuda").to(x.dtype)
    x[9] = torch.linspace(-1, 1, V, device="cuda").to(x.dtype) * 0.01
    x[10] = torch.linspace(-20, 20, V, device="cuda").to(x.dtype)
    x[11, ::2] = -float("inf")
    for k in (1, 64, 288, 1000):
        check(x, k, 1.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows", [47, 49, 81])
def test_long_rows(rows, dtype):
    """Either side of the numbers of rows from which on a row has a block."""
    V, inf = 40003, float("inf")
    g = torch.Generator("cuda").manual_seed(rows)
    x = (2.5 * torch.randn((rows, V), generator=g, device="cuda")).to(DTYPES[dtype])
    x[1] = 0.5
    x[2] = -inf
    x[3, 10:] = -inf
    x[4, 5] = float("nan")
    x[5, 7] = inf
    x[6, 1:] = torch.finfo(x.dtype).min
    x[7] = torch.randint(0, 3, (V,), generator=g, device="cuda").to(x.dtype)
    x[8, ::2] = -inf
    for k in (1, 64, 65, 288, 289):
        check(x, k, 0.7)
