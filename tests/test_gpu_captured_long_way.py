"""Backward passes captured into a CUDA graph by the long way: what a native call refuses is refused there too, and the process goes on."""
import numpy as np
import pytest
import torch

import paper_2502_01662_b200 as pkg
from paper_2502_01662_b200 import draft

pytestmark = pytest.mark.gpu


def make():
    g = torch.Generator("cuda").manual_seed(6)
    s = torch.randn((4, 2001), generator=g, device="cuda")
    top = pkg.top_logits(torch.randn((4, 2001), generator=g, device="cuda"), 12)
    return s, (top["ids"], top["values"], top["lse"], np.ones(1)), torch.rand(4, generator=g, device="cuda")     # (weights that no native call takes)


def captured(leaf, of, lists, rw, refused):
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    grad = None
    with torch.cuda.graph(graph):
        loss = pkg.distill_loss(of(leaf), *lists)
        assert "Distill" in type(loss.grad_fn).__name__ and "CppFunction" not in type(loss.grad_fn).__name__
        if refused:
            with pytest.raises(RuntimeError, match=refused):
                torch.autograd.grad(loss, leaf, rw)
        else:
            grad, = torch.autograd.grad(loss, leaf, rw)
    graph.replay()
    torch.cuda.synchronize()
    return loss, grad


def test_with_the_native_module():
    s, lists, rw = make()
    assert draft._calls()
    leaf = s.clone().requires_grad_(True)
    loss, grad = captured(leaf, lambda x: x, lists, rw, None)
    other = s.clone().requires_grad_(True)
    alive = pkg.distill_loss(other, *lists)
    want, = torch.autograd.grad(alive, other, rw, retain_graph=True)
    assert torch.equal(loss, alive) and torch.equal(grad, want)
    again, _ = captured(other, lambda x: x, lists, rw, "eager graph")
    assert torch.equal(again, alive) and torch.equal(torch.autograd.grad(alive, other, rw)[0], want)


def test_without_it(monkeypatch):
    s, lists, rw = make()
    monkeypatch.setattr(draft, "_native", False)
    leaf = s.clone().requires_grad_(True)
    loss, _ = captured(leaf, lambda x: x, lists, rw, "cannot be captured")
    want = pkg.distill_loss(leaf, *lists)
    assert torch.equal(loss, want)
    eager, = torch.autograd.grad(want, leaf, rw)
    del want
    # a student that is computed, with no other graph of the leaf alive
    fresh = s.clone().requires_grad_(True)
    _, grad = captured(fresh, lambda x: x * 1.0, lists, rw, None)
    assert torch.equal(grad, eager)
