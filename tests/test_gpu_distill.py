"""cos_distill_* against the formulas in 64 bits, against differences, and through autograd."""
import math

import numpy as np
import pytest
import torch

import paper_2502_01662_b200 as pkg
from draft_reference import DTYPES, check_grad, check_loss, distill

pytestmark = pytest.mark.gpu


def make(rows, V, dtype, lists, k, seed, whole=True, T=1.0, pad=0, shift=0, repeat=False):
    g = torch.Generator("cuda").manual_seed(seed)
    shared = 2.0 * torch.randn((rows, V), generator=g, device="cuda")
    buf = torch.zeros(rows * (V + pad) + shift, dtype=DTYPES[dtype], device="cuda")
    s = buf[shift:].view(rows, V + pad)[:, :V]
    s.copy_(shared + torch.randn((rows, V), generator=g, device="cuda"))
    ids, values, lse = [], [], []
    for _ in range(lists):
        teacher = shared + torch.randn((rows, V), generator=g, device="cuda")
        v, i = torch.topk(teacher, min(k, V), dim=1)
        if k > V or repeat:                            # the same tokens again
            v, i = torch.cat([v] * (k // v.shape[1] + 1), 1)[:, :k], torch.cat([i] * (k // i.shape[1] + 1), 1)[:, :k]
            if repeat:
                i = torch.where(torch.arange(k, device="cuda") % 3 == 0, i[:, :1], i)
        ids.append(i.int())
        values.append(v)
        lse.append(torch.logsumexp(teacher.double() / T, 1).float())
    return s, torch.stack(ids, 1).contiguous(), torch.stack(values, 1).contiguous(), torch.stack(lse, 1).contiguous() if whole else None


def reference(s, ids, values, lse, weights, T):
    host = lambda v: None if v is None else v.double().cpu().numpy()  # noqa: E731
    s, values, lse = host(s), host(values), host(lse)
    ids = ids.cpu().numpy()
    T = float(T)
    return [distill(s[r], ids[r], values[r], None if lse is None else lse[r], weights, T) for r in range(s.shape[0])], s, T


def check(s, ids, values, lse, weights, T, seed=0):
    """Loss, gradient through autograd, and the step, of one problem."""
    rows = s.shape[0]
    want, host, T64 = reference(s.detach(), ids, values, lse, weights, T)
    rw = torch.rand(rows, generator=torch.Generator("cuda").manual_seed(seed), device="cuda") + 0.25
    leaf = s.detach().requires_grad_(True)
    loss = pkg.distill_loss(leaf, ids, values, lse, weights, T)
    grad, = torch.autograd.grad(loss, leaf, rw)
    assert grad.dtype == s.dtype and grad.shape == s.shape
    alone = pkg.distill_loss(s.detach(), ids, values, lse, weights, T)
    assert torch.equal(alone, loss)
    step = pkg.distill_step(s.detach(), ids, values, rw, lse, weights, T)
    for r in range(rows):
        l, g, t, q = want[r]
        for got_l, got_g in ((loss, grad), (step["loss"], step["grad"])):
            check_loss(float(got_l[r].detach()), l, t, host.shape[1])
            check_grad(got_g[r].double().cpu().numpy(), g, q, t, host[r], T64, float(rw[r]), s.dtype)
    return step


@pytest.mark.parametrize("whole", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,V,lists,k,T", [(1, 1, 1, 1, 1.0), (2, 9, 1, 3, 0.5), (3, 100, 2, 10, 2.0), (5, 4099, 1, 64, 1.0), (2, 32000, 3, 17, 1.5), (1, 151936, 2, 32, 0.7), (300, 1003, 1, 5, 1.0),
                                             (4, 5000, 8, 128, 1.0), (2, 2000, 1, 1024, 3.0)])
def test_sizes(rows, V, lists, k, T, dtype, whole):
    weights = [float(w) for w in np.arange(1, lists + 1) / np.arange(1, lists + 1).sum()]
    check(*make(rows, V, dtype, lists, k, seed=V + k, whole=whole, T=T), weights, T)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(1, 0), (3, 5), (8, 8)])
def test_rows_that_start_anywhere(dtype, pad, shift):
    s, ids, values, lse = make(7, 3001, dtype, 2, 20, seed=pad, pad=pad, shift=shift)
    step = check(s, ids, values, lse, [0.5, 0.5], 1.0)
    rw = torch.rand(7, generator=torch.Generator("cuda").manual_seed(0), device="cuda") + 0.25
    buf = torch.full((7, 3001 + 4), 7.0, dtype=s.dtype, device="cuda")
    into = pkg.distill_step(s, ids, values, rw, lse, [0.5, 0.5], 1.0, grad=buf[:, 3:3004])
    assert torch.equal(into["grad"], step["grad"]) and bool((buf[:, :3] == 7.0).all()) and bool((buf[:, 3004:] == 7.0).all())
    inside = pkg.distill_step(s, ids, values, rw, lse, [0.5, 0.5], 1.0, grad=s)        # in place
    assert inside["grad"] is s and torch.equal(s, step["grad"]) and torch.equal(inside["loss"], step["loss"])


def test_tokens_that_come_up_again():
    for whole in (True, False):
        check(*make(4, 500, "f32", 3, 40, seed=3, whole=whole, repeat=True), [0.2, 0.3, 0.5], 1.0)
        check(*make(3, 6, "f32", 2, 50, seed=4, whole=whole), [0.5, 0.5], 1.0)


def test_empty_entries_and_rows():
    s, ids, values, lse = make(6, 3000, "bf16", 2, 16, seed=5)
    s[0] = float("nan")
    ids[0] = -1                                        # padding, with anything in it
    ids[1, 0] = -1                                     # a teacher that lists nothing
    ids[2, :, 3:] = -7
    values[3, :, 1:] = -float("inf")
    values[4] = -float("inf")
    lse[0] = float("nan")
    for l in (lse, None):
        step = check(s, ids, values, l, [0.4, 0.6], 1.0)
        assert step["loss"][[0, 4]].tolist() == [0.0, 0.0] and bool((step["grad"][[0, 4]] == 0).all())


def test_rows_of_weight_zero_have_no_gradient():
    s, ids, values, lse = make(4, 3000, "f32", 1, 16, seed=6)
    s[1, 7] = float("nan")
    rw = torch.tensor([1.0, 0.0, 0.0, -2.0], device="cuda")
    step = pkg.distill_step(s, ids, values, rw, lse)
    leaf = s.clone().requires_grad_(True)
    loss = pkg.distill_loss(leaf, ids, values, lse)
    grad, = torch.autograd.grad(loss, leaf, rw)
    loss = loss.detach()
    for g in (grad, step["grad"]):
        assert bool((g[1:3] == 0).all()) and bool((g[[0, 3]] != 0).any())
    assert math.isnan(float(loss[1])) and math.isnan(float(step["loss"][1]))
    want, _, _ = reference(s[[0, 2, 3]], ids[[0, 2, 3]], values[[0, 2, 3]], lse[[0, 2, 3]], [1.0], 1.0)
    for i, r in enumerate((0, 2, 3)):
        check_loss(float(loss[r]), want[i][0], want[i][2], 3000)
        check_loss(float(step["loss"][r]), want[i][0], want[i][2], 3000)


def test_what_is_not_finite():
    s, ids, values, lse = make(6, 2000, "f32", 1, 8, seed=7)
    s[0, 11] = float("nan")
    s[1, 11] = float("inf")
    s[2] = -float("inf")
    s[3, ids[3, 0, 2].long()] = -float("inf")          # a token that the teacher wants is ruled out
    s[4, ::2] = -float("inf")
    s[4, ids[4, 0].long()] = 1.0
    ids[5, 0, 3] = 2000                                # no token
    rw = torch.ones(6, device="cuda")
    step = pkg.distill_step(s, ids, values, rw, lse)
    leaf = s.clone().requires_grad_(True)
    loss = pkg.distill_loss(leaf, ids, values, lse)
    grad, = torch.autograd.grad(loss, leaf, rw)
    loss = loss.detach()
    for l, g in ((loss, grad), (step["loss"], step["grad"])):
        assert all(math.isnan(float(l[r])) for r in (0, 1, 2, 5)) and float(l[3]) == math.inf and math.isfinite(float(l[4]))
        assert all(bool(g[r].isnan().all()) for r in (0, 2, 5)) and bool(g[3].isfinite().all()) and bool((g[4, s[4] == -float("inf")] == 0).all())
    want, host, T = reference(s[3:5], ids[3:5], values[3:5], lse[3:5], [1.0], 1.0)
    for i in range(2):
        check_grad(step["grad"][3 + i].double().cpu().numpy(), want[i][1], want[i][3], want[i][2], host[i], T, 1.0, s.dtype)


def test_logits_in_rising_order_and_far_apart():
    V = 20001
    s = torch.stack([torch.linspace(-30, 30, V), torch.linspace(30, -30, V), torch.full((V,), -3e38)]).cuda()
    s[2, 5] = 3e38
    ids = torch.tensor([[3, V - 1, 77], [3, 0, 77], [5, 5, 5]], dtype=torch.int32, device="cuda")
    values = torch.tensor([[1.0, 2.0, 0.5]] * 3, device="cuda")
    step = pkg.distill_step(s, ids, values, torch.ones(3, device="cuda"))
    want, host, T = reference(s, ids[:, None], values[:, None], None, [1.0], 1.0)
    for r in range(3):
        # a lane of the rising row sees a new maximum with every vector: up to V / 4 / 512 + 1 = 11 of them, within the 16 of the bound
        check_loss(float(step["loss"][r]), want[r][0], want[r][2], V)
        check_grad(step["grad"][r].double().cpu().numpy(), want[r][1], want[r][3], want[r][2], host[r], T, 1.0, torch.float32)


def test_gradient_against_differences():
    """Central differences of the 64-bit loss at a few tokens, and of the library's own at a large step."""
    s, ids, values, lse = make(1, 300, "f32", 2, 10, seed=8)
    w = [0.3, 0.7]
    grad = pkg.distill_step(s, ids, values, torch.ones(1, device="cuda"), lse, w, 1.3)["grad"][0].double().cpu().numpy()
    x, t = s[0].double().cpu().numpy(), 1.3
    l64 = lambda y: distill(y, ids[0].cpu().numpy(), values[0].double().cpu().numpy(), lse[0].double().cpu().numpy(), w, t)[0]  # noqa: E731
    for i in [int(ids[0, 0, 0]), int(ids[0, 1, 3]), 5, 99, 299]:
        h = 1e-4
        up, down = x.copy(), x.copy()
        up[i] += h
        down[i] -= h
        d = (l64(up) - l64(down)) / (2 * h)
        # the third derivative of a log-sum-exp is below 1 / T^3: h^2 / 6; rounding of the difference 2^-52 * 10 / h; the gradient's own error 2^-20 of P / T
        assert abs(d - grad[i]) <= h * h / 6 + 2.0 ** -52 * 10 / h + 2.0 ** -18, (i, d, grad[i])


def test_autograd():
    s, ids, values, lse = make(12, 5000, "f32", 1, 16, seed=9)
    leaf = s.clone().requires_grad_(True)
    loss = pkg.distill_loss(2.0 * leaf, ids, values, lse).mean()       # a graph in front of it, an expanded upstream gradient
    loss.backward()
    want, host, T = reference(2.0 * s, ids, values, lse, [1.0], 1.0)
    for r in range(12):      # (doubling is exact)
        check_grad(leaf.grad[r].double().cpu().numpy() / 2.0, want[r][1], want[r][3], want[r][2], host[r], T, float(np.float32(1.0 / 12)), torch.float32)
    # an upstream that is not contiguous
    leaf2 = s.clone().requires_grad_(True)
    up = torch.rand((12, 2), device="cuda")[:, 0]
    g, = torch.autograd.grad(pkg.distill_loss(leaf2, ids, values, lse), leaf2, up)
    other, = torch.autograd.grad(pkg.distill_loss(leaf2, ids, values, lse), leaf2, up.contiguous())
    assert torch.equal(g, other)
    with torch.no_grad():
        assert not pkg.distill_loss(leaf2, ids, values, lse).requires_grad
    with pytest.raises(RuntimeError):
        first, = torch.autograd.grad(pkg.distill_loss(leaf2, ids, values, lse).sum(), leaf2, create_graph=True)
        first.sum().backward()


def test_a_student_row_that_is_broadcast():
    """One row of logits against many lists: the gradients of all of them add up in it."""
    s, ids, values, lse = make(7, 3001, "f32", 1, 20, seed=16)
    leaf = s[:1].clone().requires_grad_(True)
    loss = pkg.distill_loss(leaf.expand(7, 3001), ids, values, lse)
    rw = torch.rand(7, generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    grad, = torch.autograd.grad(loss, leaf, rw)
    want = pkg.distill_step(s[:1].repeat(7, 1), ids, values, rw, lse)
    again = pkg.distill_step(s[:1].expand(7, 3001), ids, values, rw, lse)
    assert torch.equal(want["grad"], again["grad"]) and torch.equal(want["loss"], again["loss"])
    same = s[:1].repeat(7, 1).requires_grad_(True)
    each, = torch.autograd.grad(pkg.distill_loss(same, ids, values, lse), same, rw)
    # seven terms added in some order: 6 roundings of at most the sum of their sizes
    assert bool(((grad - each.double().sum(0, keepdim=True)).abs() <= 6 * 2.0 ** -24 * each.double().abs().sum(0, keepdim=True) + 1e-37).all())


def test_rows_longer_than_shared_memory():
    check(*make(2, 700_001, "f32", 1, 64, seed=10, pad=1), [1.0], 1.0)


def test_offsets_past_32_bits():
    V, stride = 1000, (1 << 31) + 24
    s, ids, values, lse = make(3, V, "bf16", 1, 16, seed=11)
    buf = torch.empty(2 * stride + V, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((3, V), (stride, 1))
    x.copy_(s)
    rw = torch.ones(3, device="cuda")
    want = pkg.distill_step(s, ids, values, rw, lse)
    got = pkg.distill_step(x, ids, values, rw, lse, grad=x)
    assert torch.equal(got["loss"], want["loss"]) and torch.equal(x, want["grad"])


def test_calls_agree_bit_by_bit():
    s, ids, values, lse = make(30, 32000, "bf16", 4, 64, seed=12)
    rw = torch.rand(30, device="cuda")
    first = pkg.distill_step(s, ids, values, rw, lse, [0.25] * 4)
    for _ in range(5):
        again = pkg.distill_step(s, ids, values, rw, lse, [0.25] * 4)
        assert torch.equal(first["loss"], again["loss"]) and torch.equal(first["grad"], again["grad"])


def test_streams_and_graphs():
    s, ids, values, lse = make(9, 20001, "bf16", 1, 64, seed=13)
    rw = torch.rand(9, device="cuda")
    want = pkg.distill_step(s, ids, values, rw, lse)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = pkg.distill_step(s, ids, values, rw, lse, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(other["grad"], want["grad"])
    leaf = s.clone().requires_grad_(True)
    here, = torch.autograd.grad(pkg.distill_loss(leaf, ids, values, lse), leaf, rw)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                      # forward and backward on a stream of their own
        leaf = s.clone().requires_grad_(True)
        g, = torch.autograd.grad(pkg.distill_loss(leaf, ids, values, lse), leaf, rw)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(g, here)
    graphs, outs = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            outs.append(pkg.distill_step(s, ids, values, rw, lse))
        graphs.append(graph)
    s.copy_(s.flip(0))
    fresh = pkg.distill_step(s, ids, values, rw, lse)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for graph, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o["grad"], fresh["grad"]) and torch.equal(o["loss"], fresh["loss"]) for o in outs)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_many_rows(dtype):
    """Rows enough for a block each."""
    V, rows = 20001, 310
    s, ids, values, lse = make(rows, V, dtype, 2, 24, seed=15, pad=1)
    s[1, ::2] = -float("inf")
    s[1, ids[1].flatten().long()] = 1.0
    s[2] = torch.linspace(-20, 20, V, device="cuda").to(s.dtype)      # (a lane sees up to 6 new maxima: V / 8 / 512 + 1, or 11 of fp32)
    s[3] = float("nan")
    ids[3] = -1
    check(s, ids, values, lse, [0.5, 0.5], 1.0)
    s[4, 100] = float("nan")
    s[5] = -float("inf")
    s[6, 9] = float("inf")
    loss = pkg.distill_loss(s, ids, values, lse, [0.5, 0.5])
    assert loss[4:7].isnan().all() and loss[:4].isfinite().all() and loss[7:].isfinite().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_captured_backward_pass(dtype):
    """Forward and backward in a graph, replayed on other inputs; while an eager graph of the same leaf is alive the backward pass is refused, and the process goes on."""
    s, ids, values, lse = make(7, 3001, dtype, 1, 16, seed=21)
    rw = torch.rand(7, device="cuda")
    static = s.clone().requires_grad_(True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = pkg.distill_loss(static, ids, values, lse)
        grad, = torch.autograd.grad(loss, static, rw)
    for turn in range(2):
        with torch.no_grad():
            static.copy_(s.roll(turn, 0))
        graph.replay()
        leaf = s.roll(turn, 0).requires_grad_(True)
        want = pkg.distill_loss(leaf, ids, values, lse)
        assert torch.equal(loss, want) and torch.equal(grad, torch.autograd.grad(want, leaf, rw)[0])
    leaf = s.clone().requires_grad_(True)
    alive = pkg.distill_loss(leaf, ids, values, lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        inside = pkg.distill_loss(leaf, ids, values, lse)
        with pytest.raises(RuntimeError, match="eager graph"):
            torch.autograd.grad(inside, leaf, rw)
    graph.replay()
    assert torch.equal(inside, alive)
    again, = torch.autograd.grad(alive, leaf, rw)
    assert torch.equal(again, torch.autograd.grad(pkg.distill_loss(leaf, ids, values, lse), leaf, rw)[0])
