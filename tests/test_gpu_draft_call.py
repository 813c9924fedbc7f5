"""The proposer's operators called in native code against the long way through ctypes: the same outputs and the same complaints."""
import pytest
import torch

import paper_2502_01662_b200 as pkg
from paper_2502_01662_b200 import draft

pytestmark = pytest.mark.gpu


def both(monkeypatch, call):
    assert draft._calls()
    short = call()
    with monkeypatch.context() as m:
        m.setattr(draft, "_native", False)
        long = call()
    return short, long


def same(short, long):
    assert list(short) == list(long)
    for n in short:
        a, b = short[n], long[n]
        assert a.dtype is b.dtype and a.shape == b.shape and a.stride() == b.stride() and not a.requires_grad and torch.equal(torch.nan_to_num(a.float(), nan=-7.0), torch.nan_to_num(b.float(), nan=-7.0)), n


def test_sample_and_top(monkeypatch):
    g = torch.Generator("cuda").manual_seed(1)
    for x in (torch.randn((5, 3001), generator=g, device="cuda"), torch.randn((5, 3001), generator=g, device="cuda").bfloat16(), torch.randn((5, 3008), generator=g, device="cuda").half()[:, 3:3004]):
        u = torch.rand(5, generator=g, device="cuda")
        T, k = torch.full((5,), 0.7, device="cuda"), torch.tensor([0, 3, 50, 7, 1], dtype=torch.int32, device="cuda")
        p, m = torch.rand(5, generator=g, device="cuda"), torch.tensor([0.0, 0.1, 0.0, 0.2, 0.0], device="cuda")
        x[3, 5] = float("nan")
        for args in ((), (1, 50, 0.9, 0.1), (T, k, p, m), (0.0, k, 1.0, m)):
            for filtered in (False, True):
                same(*both(monkeypatch, lambda: pkg.sample(x, u, *args, filtered=filtered)))
        same(*both(monkeypatch, lambda: pkg.top_logits(x, 40)))
        same(*both(monkeypatch, lambda: pkg.top_logits(x, 3, temperature=2)))


def test_distillation(monkeypatch):
    g = torch.Generator("cuda").manual_seed(2)
    s = torch.randn((6, 2000), generator=g, device="cuda").bfloat16()
    ids = torch.randint(0, 2000, (6, 2, 9), generator=g, device="cuda").int()
    values, lse = torch.randn((6, 2, 9), generator=g, device="cuda"), torch.full((6, 2), 3.0, device="cuda")
    rw = torch.rand(6, generator=g, device="cuda")
    cases = [(ids, values, lse, [0.5, 0.5], 1.5), (ids, values, None, (0.25, 0.75), 1), (ids[:, 0].contiguous(), values[:, 0].contiguous(), lse[:, 0].contiguous(), None, 0.5),
             (ids[:, 0].contiguous(), values[:, 0].contiguous(), None, None, 2.0)]
    for a in cases:
        ids_, values_, lse_, w, T = a
        same(*both(monkeypatch, lambda: pkg.distill_step(s, ids_, values_, rw, lse_, w, T)))

        def train():
            leaf = s.detach().requires_grad_(True)
            loss = pkg.distill_loss(leaf, ids_, values_, lse_, w, T)
            assert loss.requires_grad and loss.grad_fn is not None
            grad, = torch.autograd.grad(loss, leaf, rw)
            return {"loss": loss.detach(), "grad": grad, "alone": pkg.distill_loss(s, ids_, values_, lse_, w, T)}
        same(*both(monkeypatch, train))


def test_a_student_changed_in_place_is_noticed(monkeypatch):
    s = torch.randn((3, 100), device="cuda")
    ids, values = torch.zeros((3, 2), dtype=torch.int32, device="cuda"), torch.zeros((3, 2), device="cuda")

    def change():
        leaf = s.clone().requires_grad_(True)
        mid = leaf * 1.0
        loss = pkg.distill_loss(mid, ids, values)
        mid.mul_(2.0)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.sum().backward()
    both(monkeypatch, change)


def test_what_the_library_writes_in_place_is_noticed():
    ids, values, rw = torch.zeros((3, 2), dtype=torch.int32, device="cuda"), torch.zeros((3, 2), device="cuda"), torch.ones(3, device="cuda")
    for write in (lambda t: pkg.sample(t, rw * 0.5, top_k=3, filtered=t), lambda t: pkg.distill_step(t, ids, values, rw, grad=t)):
        mid = torch.randn((3, 100), device="cuda", requires_grad=True) * 1.0
        loss = pkg.distill_loss(mid, ids, values)
        write(mid.detach())
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.sum().backward()


def test_only_once_differentiable(monkeypatch):
    s = torch.randn((3, 100), device="cuda", requires_grad=True)
    ids, values = torch.zeros((3, 2), dtype=torch.int32, device="cuda"), torch.zeros((3, 2), device="cuda")

    def twice():
        first, = torch.autograd.grad(pkg.distill_loss(s, ids, values).sum(), s, create_graph=True)
        plain, = torch.autograd.grad(pkg.distill_loss(s, ids, values).sum(), s)
        assert torch.equal(first, plain)
        with pytest.raises(RuntimeError):
            first.sum().backward()
    both(monkeypatch, twice)


def test_the_same_complaints(monkeypatch):
    x, u = torch.zeros(4, 10, device="cuda"), torch.zeros(4, device="cuda")
    ids, values = torch.zeros(4, 3, dtype=torch.int32, device="cuda"), torch.zeros(4, 3, device="cuda")
    for error, call in ((ValueError, lambda: pkg.sample(x.cpu(), u)), (ValueError, lambda: pkg.sample(x, u.double())), (ValueError, lambda: pkg.sample(x, u, top_k=u)),
                        (pkg.CosVerifyError, lambda: pkg.sample(x, u, -1.0)), (pkg.CosVerifyError, lambda: pkg.top_logits(x, 2, 0.0)), (ValueError, lambda: pkg.top_logits(x, 11)),
                        (ValueError, lambda: pkg.distill_loss(x, ids.long(), values)), (pkg.CosVerifyError, lambda: pkg.distill_loss(x, ids, values, temperature=0.0)),
                        (pkg.CosVerifyError, lambda: pkg.distill_loss(x.clone().requires_grad_(True), ids, values, temperature=0.0)), (ValueError, lambda: pkg.distill_step(x, ids, values, u[:2])),
                        (pkg.CosVerifyError, lambda: pkg.distill_step(x, ids, values, u, weights=[-1.0]))):
        def check():
            with pytest.raises(error):
                call()
        both(monkeypatch, check)


def test_calls_of_several_threads():
    """Calls at once whose launches take different amounts of shared memory: none fails, all results are those of calls one by one."""
    import threading
    sizes = [(2, 900), (3, 60000), (40, 32000), (5, 9000)]
    rows = [(torch.randn(n, V, device="cuda", generator=torch.Generator("cuda").manual_seed(V)), torch.rand(n, device="cuda")) for n, V in sizes]
    def calls(x, u):
        top = pkg.top_logits(x, 20)
        step = pkg.distill_step(x, top["ids"], top["values"] + 0.1, u, top["lse"])
        return pkg.sample(x, u, 0.9, 0, 0.9)["tokens"], top["ids"], step["grad"], step["loss"]
    want = [calls(x, u) for x, u in rows]
    wrong = []
    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(100):
                    got = calls(*rows[i])
                    if not all(torch.equal(a, b) for a, b in zip(got, want[i])):
                        wrong.append(i)
        except Exception as e:  # noqa: BLE001
            wrong.append(e)
    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(rows))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong[:3]


@pytest.mark.parametrize("k", [2 ** 31 - 1, 2 ** 31, 2 ** 32 + 5, 2 ** 70, -(2 ** 31), -(2 ** 32) + 5])
def test_numbers_beyond_32_bits_are_no_limit(k):
    x, u = torch.randn(3, 500, device="cuda"), torch.rand(3, device="cuda")
    want, got = pkg.sample(x, u), pkg.sample(x, u, top_k=k)
    assert all(torch.equal(got[n], want[n]) for n in want) and (got["kept"] == 500).all()


def test_more_rows_than_32_bits():
    x = torch.zeros((1, 4), device="cuda").expand(2 ** 31, 4)
    with pytest.raises(ValueError):
        pkg.top_logits(x, 2)
