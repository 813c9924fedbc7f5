"""What goes wrong inside a call of the proposer's operators is an error in Python, by the native call and by the long way: lists of inference mode, hooks on saved tensors, no memory."""
import pytest
import torch
import torch.autograd.forward_ad as forward_ad
from torch.utils.checkpoint import checkpoint

import paper_2502_01662_b200 as pkg
from paper_2502_01662_b200 import draft

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["native", "long"])
def way(request, monkeypatch):
    assert draft._calls()
    if request.param == "long":
        monkeypatch.setattr(draft, "_native", False)
    return request.param


def make():
    g = torch.Generator("cuda").manual_seed(4)
    s = torch.randn((5, 3001), generator=g, device="cuda")
    top = pkg.top_logits(s + torch.randn((5, 3001), generator=g, device="cuda"), 16)
    return s, top["ids"], top["values"], top["lse"], torch.rand(5, generator=g, device="cuda")


def test_lists_of_inference_mode(way):
    s, ids, values, lse, rw = make()
    with torch.inference_mode():
        top = pkg.top_logits(s, 16)
    inside = top["ids"], top["values"], top["lse"]
    leaf = s.clone().requires_grad_(True)
    for lists in (inside, (inside[0], values, lse), (ids, values, inside[2])):
        with pytest.raises(RuntimeError, match="[Ii]nference"):
            pkg.distill_loss(leaf, *lists)
    # where nothing is kept for a backward pass they are lists like others, and so are copies of them
    copies = [t.clone() for t in inside]
    loss = pkg.distill_loss(leaf, *copies)
    assert torch.equal(pkg.distill_loss(s, *inside), loss)
    step, other = (pkg.distill_step(s, *lists[:2], rw, lists[2]) for lists in (inside, copies))
    assert torch.equal(step["loss"], other["loss"]) and torch.equal(step["grad"], other["grad"])
    assert bool(torch.autograd.grad(loss, leaf, rw)[0].isfinite().all())


def test_a_student_with_a_tangent_and_a_gradient(way):
    s, ids, values, lse, _ = make()
    with forward_ad.dual_level():
        with pytest.raises(RuntimeError, match="jvp"):
            pkg.distill_loss(forward_ad.make_dual(s.clone().requires_grad_(True), torch.ones_like(s)), ids, values, lse)


def test_hooks_on_saved_tensors(way):
    s, ids, values, lse, rw = make()
    leaf = s.clone().requires_grad_(True)
    want, = torch.autograd.grad(pkg.distill_loss(leaf, ids, values, lse), leaf, rw)

    def refuse(t):
        raise ValueError("not this one")
    with torch.autograd.graph.saved_tensors_hooks(refuse, lambda t: t):
        with pytest.raises(ValueError, match="not this one"):
            pkg.distill_loss(leaf, ids, values, lse)
    with torch.autograd.graph.save_on_cpu():
        loss = pkg.distill_loss(leaf, ids, values, lse)
    assert torch.equal(torch.autograd.grad(loss, leaf, rw)[0], want)
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, refuse):
        loss = pkg.distill_loss(leaf, ids, values, lse)
    with pytest.raises(ValueError, match="not this one"):
        torch.autograd.grad(loss, leaf, rw)


def test_the_last_operation_of_a_checkpoint(way):
    s, ids, values, lse, rw = make()

    def forward(x):
        return pkg.distill_loss(2.0 * x, ids, values, lse)
    leaf = s.clone().requires_grad_(True)
    want, = torch.autograd.grad(forward(leaf), leaf, rw)
    for _ in range(2):
        loss = checkpoint(forward, leaf, use_reentrant=False)
        grad, = torch.autograd.grad(loss, leaf, rw)
        assert torch.equal(grad, want)


def test_no_memory(way):
    s, ids, values, lse, rw = make()
    leaf = s.clone().requires_grad_(True)
    u = rw.clone()
    alive = pkg.distill_loss(leaf, ids, values, lse)
    calls = [lambda: pkg.sample(s, u), lambda: pkg.sample(s, u, 0.7, 50, 0.9, filtered=True), lambda: pkg.top_logits(s, 16), lambda: pkg.distill_loss(s, ids, values, lse),
             lambda: pkg.distill_loss(leaf, ids, values, lse), lambda: pkg.distill_step(s, ids, values, rw, lse), lambda: torch.autograd.grad(alive, leaf, rw, retain_graph=True)]
    want = [call() for call in calls]
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    filler = []
    try:
        torch.cuda.set_per_process_memory_fraction(0.0)      # (of this process and torch's allocator alone: no new segment)
        for size in (1 << 20, 1 << 9):                       # what is left of the segments there are, down to the smallest pieces
            with pytest.raises(torch.OutOfMemoryError):
                while len(filler) < 1 << 17:
                    filler.append(torch.empty(size, dtype=torch.uint8, device="cuda"))
        for call in calls:
            with pytest.raises(torch.OutOfMemoryError):
                call()
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)
        filler.clear()
    flat = lambda v: list(v.values()) if isinstance(v, dict) else list(v) if isinstance(v, tuple) else [v]  # noqa: E731
    for call, before in zip(calls, want):
        assert all(torch.equal(a, b) for a, b in zip(flat(call()), flat(before)))


def test_a_student_with_a_tangent_alone(way):
    """No gradient is wanted, and none may be lost: neither in a graph nor without one."""
    s, ids, values, lse, _ = make()
    want = pkg.distill_loss(s, ids, values, lse)
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(s, torch.ones_like(s))
        for grad in (True, False):
            with torch.set_grad_enabled(grad), pytest.raises(NotImplementedError, match="forward mode"):
                pkg.distill_loss(dual, ids, values, lse)
        assert torch.equal(pkg.distill_loss(forward_ad.unpack_dual(dual).primal, ids, values, lse), want)
    assert torch.equal(pkg.distill_loss(s, ids, values, lse), want)
