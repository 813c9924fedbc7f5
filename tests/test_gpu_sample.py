"""cos_sample against its definition in 64 bits: types, sizes, limits, masks, ties, strides, streams, graphs."""
import numpy as np
import pytest
import torch

import paper_2502_01662_b200 as pkg
from draft_reference import DTYPES, check_samples

pytestmark = pytest.mark.gpu


def make(rows, V, dtype, seed, sigma=2.5, pad=0, shift=0):
    g = torch.Generator("cuda").manual_seed(seed)
    buf = torch.zeros(rows * (V + pad) + shift, dtype=DTYPES[dtype], device="cuda")
    x = buf[shift:].view(rows, V + pad)[:, :V]
    x.copy_(sigma * torch.randn((rows, V), generator=g, device="cuda"))
    return x, torch.rand(rows, generator=g, device="cuda")


def run(x, u, T=1.0, k=0, p=1.0, least=0.0, **kw):
    kw.setdefault("filtered", True)
    out = pkg.sample(x, u, T, k, p, least, **kw)
    host = lambda v: v.cpu().numpy() if isinstance(v, torch.Tensor) else v  # noqa: E731
    check_samples(x, u, host(T), host(k), host(p), host(least), out)
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,V", [(1, 1), (3, 2), (5, 7), (2, 8), (4, 65), (9, 1000), (3, 4099), (2, 32000), (1, 151936), (150, 515), (33, 20001)])
def test_sizes_and_limits(rows, V, dtype):
    x, u = make(rows, V, dtype, seed=rows * 31 + V)
    for T, k, p, least in ((1.0, 0, 1.0, 0.0), (0.7, 50, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (0.8, 40, 0.95, 0.0), (1.2, 0, 1.0, 0.05), (1.0, 300, 0.8, 0.02), (0.0, 7, 0.5, 0.1), (1.0, 1, 1.0, 0.0)):
        run(x, u, T, k, p, least)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (3, 5), (8, 8)])
def test_rows_that_start_anywhere(dtype, pad, shift):
    x, u = make(6, 5003, dtype, seed=pad * 10 + shift, pad=pad, shift=shift)
    before = x.clone()
    a = run(x, u, 0.9, 100, 0.9, 0.01)
    assert torch.equal(x, before)
    # into a tensor of another alignment, whose other entries stay
    buf = torch.full((6, 5003 + 4), 7.0, dtype=x.dtype, device="cuda")
    b = run(x, u, 0.9, 100, 0.9, 0.01, filtered=buf[:, 3:5006])
    assert torch.equal(a["tokens"], b["tokens"]) and torch.equal(a["filtered"], b["filtered"])
    assert bool((buf[:, :3] == 7.0).all()) and bool((buf[:, 5006:] == 7.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place(dtype):
    for pad in (0, 5):
        x, u = make(5, 30001, dtype, seed=9 + pad, pad=pad)
        want = run(x, u, 0.8, 60, 0.9, 0.0)
        rest = x.as_strided((5, pad), (30001 + pad, 1), 30001).clone()
        got = pkg.sample(x, u, 0.8, 60, 0.9, 0.0, filtered=x)
        assert got["filtered"] is x and torch.equal(x, want["filtered"]) and torch.equal(got["tokens"], want["tokens"])
        assert torch.equal(x.as_strided((5, pad), (30001 + pad, 1), 30001), rest)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_rows_of_their_own_parameters(dtype):
    rows, V = 48, 9001
    x, u = make(rows, V, dtype, seed=77)
    g = np.random.default_rng(5)
    T = torch.tensor(np.where(g.random(rows) < 0.2, 0.0, g.uniform(0.05, 3.0, rows)), dtype=torch.float32, device="cuda")
    k = torch.tensor(np.where(g.random(rows) < 0.3, 0, g.integers(-2, 3000, rows)), dtype=torch.int32, device="cuda")
    p = torch.tensor(np.where(g.random(rows) < 0.3, 1.0, g.uniform(0.0, 1.2, rows)), dtype=torch.float32, device="cuda")
    m = torch.tensor(np.where(g.random(rows) < 0.5, 0.0, g.uniform(-0.2, 1.2, rows)), dtype=torch.float32, device="cuda")
    run(x, u, T, k, p, m)


def test_one_row_for_many_draws():
    """A row that is broadcast: a uniform and limits of its own for each draw."""
    x, _ = make(1, 5001, "bf16", seed=31)
    g = torch.Generator("cuda").manual_seed(31)
    u = torch.rand(64, generator=g, device="cuda")
    k = torch.randint(0, 300, (64,), generator=g, device="cuda").int()
    run(x.expand(64, 5001), u, 0.9, k, 0.95)
    with pytest.raises(pkg.CosVerifyError):
        pkg.sample(x.expand(64, 5001), u, filtered=x.expand(64, 5001))


def test_bad_parameters_of_rows_are_reported():
    x, u = make(6, 500, "f32", seed=3)
    T = torch.tensor([1.0, -1.0, float("nan"), 0.5, float("inf"), 1e-30], device="cuda")
    out = run(x, u, T)
    assert out["row_status"].tolist() == [0, 1, 1, 0, 0, 0]
    nan = torch.full((6,), float("nan"), device="cuda")
    out = pkg.sample(x, u, 1.0, 0, nan, nan)           # no limit, no minimum
    assert out["kept"].tolist() == [500] * 6 and bool((out["tokens"] >= 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [300, 5000, 70001])
def test_ties(dtype, V):
    """Few different values, so that borders lie among thousands of equal tokens: the lowest indices of them are kept."""
    g = torch.Generator("cuda").manual_seed(V)
    x = torch.randint(0, 3, (4, V), generator=g, device="cuda").to(DTYPES[dtype])
    u = torch.rand(4, generator=g, device="cuda")
    for k, p in ((7, 1.0), (V // 2, 1.0), (0, 0.3), (0, 0.999), (V // 2, 0.7), (3, 0.5)):
        run(x, u, 1.0, k, p)
    flat = torch.full((2, V), 1.25, dtype=DTYPES[dtype], device="cuda")
    for k, p in ((5, 1.0), (0, 0.5), (V - 1, 0.25), (V // 3, 0.999)):
        run(flat, u[:2], 0.7, k, p)


def test_equal_zeros():
    x = torch.zeros((2, 64), device="cuda")
    x[0, ::2] = -0.0
    x[1, :32] = -0.0
    out = run(x, torch.tensor([0.6, 0.99], device="cuda"), 1.0, 10)
    assert out["kept"].tolist() == [10, 10] and bool((out["filtered"][:, :10] == 0).all())
    assert pkg.sample(x, torch.zeros(2, device="cuda"), 0.0)["tokens"].tolist() == [0, 0]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_masks(dtype):
    V = 6001
    x, u = make(9, V, dtype, seed=8)
    low = torch.finfo(x.dtype).min
    inf = float("inf")
    x[0, :] = -inf                       # nothing left
    x[1, :] = -inf
    x[1, 4321] = 3.0                     # one token
    x[2, 1:] = low                       # the type's lowest value
    x[3, :] = low                        # ... everywhere
    x[4, 17] = float("nan")
    x[5, 6000] = inf
    x[6, ::2] = -inf
    x[7, 100:] = -inf
    x[8, :] = torch.where(torch.arange(V, device="cuda") % 3 == 0, torch.tensor(low, device="cuda"), x[8].float()).to(x.dtype)
    for T, k, p, least in ((1.0, 0, 1.0, 0.0), (0.7, 30, 0.9, 0.0), (0.0, 0, 1.0, 0.0), (2.0, 0, 0.99, 0.001), (1.0, 5000, 1.0, 0.0)):
        out = run(x, u, T, k, p, least)
        assert out["row_status"].tolist() == [1, 0, 0, 0, 1, 1, 0, 0, 0]


def test_uniforms_at_and_beyond_their_bounds():
    x, _ = make(8, 3001, "f32", seed=4)
    x[:] = x[0]
    x[:, 0] = -float("inf")
    u = torch.tensor([0.0, 1.0 - 2.0 ** -24, 1.0, 2.0, -1.0, float("nan"), 2.0 ** -24, 0.5], device="cuda")
    out = run(x, u, 1.0, 20)
    kept = torch.nonzero(out["filtered"][0] > -float("inf")).flatten()
    t = out["tokens"].tolist()
    assert t[0] == t[4] == t[5] == int(kept[0]) and t[1] == t[2] == t[3] == int(kept[-1])


@pytest.mark.parametrize("T", [1e-20, 1e-3, 0.05, 30.0, 1e6, 1e30])
def test_extreme_temperatures(T):
    for dtype in ("f32", "bf16"):
        x, u = make(3, 12001, dtype, seed=6)
        for k, p, least in ((0, 1.0, 0.0), (40, 1.0, 0.0), (0, 0.9, 0.0), (3000, 0.5, 0.0), (0, 1.0, 0.5)):
            run(x, u, T, k, p, least)


def test_logits_far_apart():
    x = torch.zeros((2, 4000), device="cuda")
    x[0] = torch.linspace(-3e38, 3e38, 4000, device="cuda")
    x[1] = torch.linspace(-1e4, 1e4, 4000, device="cuda")
    u = torch.tensor([0.3, 0.9], device="cuda")
    for k, p in ((0, 1.0), (1000, 1.0), (0, 0.9), (3999, 0.9999)):
        run(x, u, 1.0, k, p)
        run(x, u, 1e4, k, p)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_longer_than_shared_memory(dtype):
    x, u = make(2, 1_200_007, dtype, seed=12, pad=1)
    for k, p, least in ((0, 1.0, 0.0), (100, 0.9, 0.0), (0, 0.5, 0.0), (0, 1.0, 0.1)):
        run(x, u, 1.0, k, p, least)
    want = run(x, u, 1.0, 100, 0.9)
    pkg.sample(x, u, 1.0, 100, 0.9, filtered=x)
    assert torch.equal(x, want["filtered"])


def test_a_row_of_millions():
    """More vectors of a lane than fit into a word of bits."""
    x, u = make(1, 5_000_011, "bf16", seed=14, sigma=4.0)
    for k, p in ((0, 1.0), (0, 0.7), (2000, 0.9)):
        run(x, u, 1.0, k, p)


def test_offsets_past_32_bits():
    V, stride = 1000, (1 << 31) + 24
    buf = torch.empty(2 * stride + V, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((3, V), (stride, 1))
    x.copy_(torch.randn((3, V), generator=torch.Generator("cuda").manual_seed(1), device="cuda"))
    u = torch.tensor([0.1, 0.5, 0.9], device="cuda")
    out = run(x, u, 1.0, 50, 0.9)
    again = pkg.sample(x, u, 1.0, 50, 0.9, filtered=x)
    assert torch.equal(x, out["filtered"]) and torch.equal(again["tokens"], out["tokens"])


def test_more_rows_than_the_device_has_places():
    x, u = make(3001, 257, "bf16", seed=2)
    run(x, u, 0.9, 20, 0.8)


def test_calls_agree_bit_by_bit():
    x, u = make(40, 128256, "bf16", seed=5)
    first = pkg.sample(x, u, 1.0, 0, 0.9, filtered=True)
    for _ in range(5):
        again = pkg.sample(x, u, 1.0, 0, 0.9, filtered=True)
        assert all(torch.equal(first[n], again[n]) for n in first)


def test_streams_and_graphs():
    x, u = make(7, 20001, "bf16", seed=21)
    want = run(x, u, 0.8, 50, 0.9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = pkg.sample(x, u, 0.8, 50, 0.9, filtered=True, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(other[n], want[n]) for n in want)
    # two graphs of it, replayed on two streams at once with new inputs
    graphs, outs, xs, us = [], [], [], []
    for i in range(2):
        xs.append(x.clone())
        us.append(u.clone())
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            outs.append(pkg.sample(xs[i], us[i], 0.8, 50, 0.9, filtered=True))
        graphs.append(g)
    for i in range(2):
        y, v = make(7, 20001, "bf16", seed=22 + i)
        xs[i].copy_(y)
        us[i].copy_(v)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
    torch.cuda.synchronize()
    for i in range(2):
        check_samples(xs[i], us[i], 0.8, 50, 0.9, 0.0, outs[i])


def test_the_current_device_stays():
    assert torch.cuda.current_device() == 0
    x, u = make(2, 100, "f32", seed=1)
    run(x, u)
    assert torch.cuda.current_device() == 0


def test_every_token_is_drawn_as_often_as_its_weight_says():
    V, N = 11, 1 << 15
    x = torch.tensor([[0.3, 1.0, -float("inf"), 2.0, 0.0, 1.5, -1.0, 2.0, 0.7, -2.0, 1.1]], device="cuda").expand(N, V).contiguous()
    u = (torch.arange(N, device="cuda") + 0.5) / N            # every part of [0, 1) alike
    out = pkg.sample(x, u, 0.8, 6, 0.9)
    w = np.exp((x[0].double().cpu().numpy() - 2.0) / 0.8)
    line = np.argsort(-w, kind="stable")[:6]
    n = int(np.count_nonzero(np.concatenate(([0.0], np.cumsum(w[line])[:-1])) < np.float32(0.9) * w[line].sum()))
    law = np.zeros(V)
    law[line[:n]] = w[line[:n]] / w[line[:n]].sum()
    counts = np.bincount(out["tokens"].cpu().numpy(), minlength=V)
    assert np.all(np.abs(counts - N * law) <= 1.0 + 1e-6), (counts, N * law)     # N law uniforms lie in a token's part, to within one at either end


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_many_long_rows(dtype):
    """Rows enough for a block each, longer than its shared memory: masks, ties and rows that are not finite among ordinary ones, unaligned."""
    rows, V = 61, 40001
    x, u = make(rows, V, dtype, seed=17, pad=1)
    inf = float("inf")
    g = torch.Generator("cuda").manual_seed(18)
    x[1] = 0.5
    x[2] = -inf
    x[3, 10:] = -inf
    x[4, 5] = float("nan")
    x[5, 7] = inf
    x[6] = torch.finfo(x.dtype).min
    x[7, 1:] = torch.finfo(x.dtype).min
    x[8] = torch.randint(0, 3, (V,), generator=g, device="cuda").to(x.dtype)
    x[9] = torch.linspace(-20, 20, V, device="cuda").to(x.dtype)
    x[10, ::2] = -inf
    for T, k, p, least in ((1.0, 50, 1.0, 0.0), (0.7, 288, 0.9, 0.0), (1.3, 1, 1.0, 0.0), (0.9, 100, 0.5, 0.05), (1.0, 289, 0.9, 0.0)):
        run(x, u, T, k, p, least)
    want = run(x, u, 0.8, 60, 0.95, 0.01)
    kept = x.as_strided((rows, 1), (V + 1, 1), V).clone()
    got = pkg.sample(x, u, 0.8, 60, 0.95, 0.01, filtered=x)
    assert torch.equal(torch.nan_to_num(x.float(), nan=-7.0), torch.nan_to_num(want["filtered"].float(), nan=-7.0)) and torch.equal(got["tokens"], want["tokens"])
    assert torch.equal(x.as_strided((rows, 1), (V + 1, 1), V), kept)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,V", [(15, 40001), (17, 20001), (39, 40001)])
def test_few_long_rows(rows, V, dtype):
    """Either side of the numbers of rows from which on a row has a block: the largest logit and a few, ties and masks among them, in place."""
    x, u = make(rows, V, dtype, seed=rows, pad=3)
    inf = float("inf")
    x[1] = -2.0
    x[2] = -inf
    x[3, : V - 1] = -inf
    x[4, 9] = float("nan")
    x[5, 11] = inf
    x[6] = torch.finfo(x.dtype).min
    x[7, 100::1000] = 60.0
    x[8, V - 1] = 60.0
    x[9, 0] = 60.0
    x[10, 1::2] = -inf
    for T, k, p, least in ((0.0, 0, 1.0, 0.0), (0.0, 20, 0.3, 0.9), (0.8, 64, 0.9, 0.0), (0.8, 65, 1.0, 0.01)):
        run(x, u, T, k, p, least)
    for T, k in ((0.0, 0), (0.8, 64)):
        y = x.as_strided((rows, V + 3), (V + 3, 1), 0).clone()
        rest = y[:, V:].clone()
        want = run(x, u, T, k)
        got = pkg.sample(y[:, :V], u, T, k, filtered=y[:, :V])
        assert torch.equal(torch.nan_to_num(y[:, :V].float(), nan=-7.0), torch.nan_to_num(want["filtered"].float(), nan=-7.0)) and torch.equal(got["tokens"], want["tokens"])
        assert torch.equal(y[:, V:], rest)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,V", [(1, 3001), (300, 3001), (3, 16001), (2, 131071), (40, 131071)])
def test_limits_far_down_the_line(rows, V, dtype):
    """Flat rows, whose limit by mass lies behind thousands of tokens: uniforms all over the mass, ties at the limit, min-p before and behind it."""
    g = torch.Generator("cuda").manual_seed(rows + V)
    x = (1.5 * torch.rand((rows, V), generator=g, device="cuda")).to(DTYPES[dtype])
    x[0, : V // 2] = 0.75  # (a limit among equals, of more than a list holds)
    x[rows // 2, ::3] = -float("inf")
    u = (torch.arange(rows, device="cuda") + 0.5) / rows
    for T, k, p, least in ((1.0, 0, 0.5, 0.0), (0.3, 0, 0.9, 0.0), (1.0, 2 * V // 3, 0.6, 0.0), (1.0, 0, 0.7, 0.5), (0.7, 0, 0.2, 0.01), (1.0, 2000, 0.9999, 0.0)):
        run(x, u, T, k, p, least)


@pytest.mark.parametrize("k,p,least", [(0, 1.0, 1.0), (0, 1.0, 0.5), (20, 1.0, 1.0), (20, 0.4, 1.0), (0, 0.01, 1.0), (300, 0.9, 0.0)])
def test_a_temperature_without_an_end(k, p, least):
    """Every token weighs the same, and min-p takes none."""
    x, u = make(50, 2000, "f32", seed=5)
    x[1, ::2] = -float("inf")
    out = pkg.sample(x, u, float("inf"), k, p, least)
    for n in range(50):
        row = x[n].cpu().numpy().astype(np.float64)
        line = np.argsort(-row, kind="stable")[: int(np.isfinite(row).sum())]
        line = line[: k] if k else line
        total = len(line)
        line = np.sort(line[: int(np.ceil(np.float64(np.float32(p)) * total))])
        assert int(out["kept"][n]) == len(line) and int(out["row_status"][n]) == 0
        at = np.float64(np.float32(u[n].item())) * len(line)
        assert abs(at - round(at)) > 1e-6  # (no uniform lies on a border)
        assert int(out["tokens"][n]) == line[int(np.floor(at))]
        assert abs(float(out["prob"][n]) - 1.0 / len(line)) <= 2.0 ** -24 / len(line)
