"""A proposer's operators as they are used together: drafts drawn under limits, verified as drawn, and a proposer taught from the models' top logits."""
import numpy as np
import pytest
import torch

import paper_2502_01662_b200 as pkg
from oracle import cos_oracle as orc
from paper_2502_01662_b200 import scheduler as sch

from draft_reference import check_grad, check_loss, check_samples, distill, top_of
from test_scheduler import oracle_verify, oracle_verify_n
from test_scheduler_propose import NumpyProposer

pytestmark = pytest.mark.gpu

WE = orc.COMBINE_PROB_ENSEMBLE


@pytest.mark.parametrize("T,limits", [(0.8, dict(top_k=40, top_p=0.9)), (1.0, dict(min_p=0.05)), (0.0, {}), (0.9, {})])
def test_the_schedulers_on_the_gpu_are_those_on_the_oracle(T, limits):
    V, N = 4099, 150

    def two(verify, propose):
        models = sch.make_table_models(2, V, contexts=64, seed=33, sigma=2.5, rho=0.85)
        return sch.AlternateProposal(models, (4, 2), T, verify, propose_seed=3, verify_seed=4, propose=propose).generate([1, 2, 3], N)[0]

    def three(verify, propose):
        models = sch.make_table_models(3, V, contexts=64, seed=41, sigma=2.0, rho=0.9)
        return sch.CollaborativeSpeculation(models, (3, 2, 1), T, verify, propose_seed=8, verify_seed=9, propose=propose).generate([4, 4], N)[0]

    for run, w, cpu in ((two, (0.5, 0.5), oracle_verify(WE, (0.5, 0.5), T, V)), (three, (0.5, 0.3, 0.2), oracle_verify_n(3, WE, (0.5, 0.3, 0.2), T, V))):
        gpu = sch.gpu_verify(WE, w, T, V)
        try:
            got = run(gpu, sch.GpuProposer(T, **limits))
        finally:
            gpu.close()
        assert got == run(cpu, NumpyProposer(T, **limits))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_draft_verify_and_teach(dtype):
    n, B, gamma, V, T, weights = 2, 24, 4, 8003, 0.8, (0.4, 0.6)
    P = gamma + 1
    g = torch.Generator("cuda").manual_seed(77)
    shared = 2.0 * torch.randn((1, B, P, V), generator=g, device="cuda")
    logits = (shared + torch.randn((n, B, P, V), generator=g, device="cuda")).to(dtype)
    before = logits.clone()
    drafts = torch.empty((B, gamma), dtype=torch.int32, device="cuda")
    # model 0 proposes, position by position, in rows that lie P * V apart; what it could not have drawn is ruled out in place
    for j in range(gamma):
        u = torch.rand(B, generator=g, device="cuda")
        got = pkg.sample(logits[0, :, j], u, T, 50, 0.95, 0.0, filtered=logits[0, :, j])
        drafts[:, j] = got["tokens"]
        check_samples(before[0, :, j], u, T, 50, 0.95, 0.0, {**got, "filtered": logits[0, :, j]})
    assert torch.equal(logits[1], before[1]) and torch.equal(logits[0, :, gamma], before[0, :, gamma])
    v = pkg.CosVerifier(n, WE, weights, T, gamma, V, B, dtype)
    try:
        out = v.run(logits, drafts, torch.zeros(B, dtype=torch.int32, device="cuda"), 5, 6, diag=True, lse=True)
        torch.cuda.synchronize()
    finally:
        v.close()
    assert not bool((out["row_status"] & (pkg.COS_ROW_NONFINITE | pkg.COS_ROW_Q_ZERO | pkg.COS_ROW_BAD_DRAFT)).any())
    # q of the verification is the law of the draw
    q = torch.softmax(logits[0, :, :gamma].double() / T, -1).gather(2, drafts[:, :, None].long())[..., 0]
    assert torch.allclose(out["diag"][:, :gamma, 2].double(), q, rtol=1e-5, atol=1e-30)
    # the models' top logits at the verified positions, and a student that learns from them
    rows = B * P
    tops = [pkg.top_logits(logits[i].view(rows, V), 32, temperature=T) for i in range(n)]
    host = [logits[i].view(rows, V).double().cpu().numpy() for i in range(n)]
    for i in range(n):
        assert torch.allclose(tops[i]["lse"], out["lse"].view(rows, n)[:, i], rtol=1e-5, atol=1e-5)
        for r in range(0, rows, 17):
            values, ids, _ = top_of(host[i][r], 32, T)
            assert np.array_equal(tops[i]["ids"][r].cpu().numpy(), ids) and np.array_equal(tops[i]["values"][r].double().cpu().numpy(), values)
    ids, values, lse = (torch.stack([t[k] for t in tops], 1).contiguous() for k in ("ids", "values", "lse"))
    student = before[0].view(rows, V).clone().requires_grad_(True)
    loss = pkg.distill_loss(student, ids, values, lse, weights, T)
    grad, = torch.autograd.grad(loss.mean(), student)
    s = student.detach().double().cpu().numpy()
    for r in range(0, rows, 17):
        l, want, t, q64 = distill(s[r], ids[r].cpu().numpy(), values[r].double().cpu().numpy(), lse[r].double().cpu().numpy(), weights, T)
        check_loss(float(loss[r].detach()), l, t, V)
        check_grad(grad[r].double().cpu().numpy(), want, q64, t, s[r], T, float(np.float32(1.0 / rows)), dtype)
