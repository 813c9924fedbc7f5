"""The proposer's operators: what they compute in plain torch, and the cases on which they are measured.

  sample        a token for each row of logits from given uniforms, at a temperature, after top-k, top-p and min-p
  top           the k largest logits of each row, in order, with the log-sum-exp of the row: a teacher's side of distillation
  loss          the divergence of a student from the mixture of its teachers' top logits, forward and (through autograd) backward
  step          the same divergence and its gradient for given row weights in one pass

`run` computes a case in plain torch, or, where `own` is set, by the calls of this repository's package.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # one draft token of one request: where the latency of a call counts
        {"name": "sample_1x152k_bf16", "op": "sample", "rows": 1, "vocab": 151936, "dtype": "bf16", "law": "zipf", "temperature": 0.7, "top_k": 50, "top_p": 0.9, "min_p": 0.0,
         "mixed": False, "filtered": False, "ruled_out": 0.0, "pad": 0},
        # a serving batch whose requests have parameters of their own (greedy ones among them); the filtered logits are what the verification takes as q
        {"name": "sample_32x128k_bf16_mixed", "op": "sample", "rows": 32, "vocab": 128256, "dtype": "bf16", "law": "gauss", "temperature": 1.0, "top_k": 0, "top_p": 1.0, "min_p": 0.0,
         "mixed": True, "filtered": True, "ruled_out": 0.0, "pad": 0},
        # a large batch, the whole vocabulary
        {"name": "sample_64x256k_bf16", "op": "sample", "rows": 64, "vocab": 256000, "dtype": "bf16", "law": "zipf", "temperature": 1.0, "top_k": 0, "top_p": 1.0, "min_p": 0.0,
         "mixed": False, "filtered": False, "ruled_out": 0.0, "pad": 0},
        # rows that start anywhere, a grammar that rules out half of the tokens, fp32
        {"name": "sample_7x50001_f32_odd", "op": "sample", "rows": 7, "vocab": 50001, "dtype": "f32", "law": "gauss", "temperature": 0.9, "top_k": 0, "top_p": 0.95, "min_p": 0.02,
         "mixed": False, "filtered": True, "ruled_out": 0.5, "pad": 3},
        # the teacher's lists for a training batch
        {"name": "top64_512x128k_bf16", "op": "top", "rows": 512, "vocab": 128256, "dtype": "bf16", "law": "gauss", "k": 64, "temperature": 1.0, "ruled_out": 0.0, "pad": 0},
        # and for the positions of a few verified rows
        {"name": "top256_8x32k_f32", "op": "top", "rows": 8, "vocab": 32000, "dtype": "f32", "law": "zipf", "k": 256, "temperature": 2.0, "ruled_out": 0.1, "pad": 1},
        # a short sequence
        {"name": "loss_16x32k_f32", "op": "loss", "rows": 16, "vocab": 32000, "dtype": "f32", "lists": 1, "k": 32, "temperature": 1.0, "whole": True, "backward": True, "padded": 0.0, "pad": 0},
        # a training batch
        {"name": "loss_1024x128k_bf16", "op": "loss", "rows": 1024, "vocab": 128256, "dtype": "bf16", "lists": 1, "k": 64, "temperature": 1.0, "whole": True, "backward": True, "padded": 0.1, "pad": 0},
        # two teachers, the ensemble that the verification accepts against
        {"name": "loss_255x152k_f16_two", "op": "loss", "rows": 255, "vocab": 151936, "dtype": "f16", "lists": 2, "k": 32, "temperature": 0.7, "whole": True, "backward": True, "padded": 0.0, "pad": 0},
        # validation: the loss alone
        {"name": "loss_512x32k_bf16_eval", "op": "loss", "rows": 512, "vocab": 32000, "dtype": "bf16", "lists": 1, "k": 64, "temperature": 2.0, "whole": False, "backward": False, "padded": 0.0, "pad": 0},
        # a training step that has its row weights in hand
        {"name": "step_2048x32k_bf16", "op": "step", "rows": 2048, "vocab": 32000, "dtype": "bf16", "lists": 1, "k": 64, "temperature": 1.0, "whole": False, "backward": True, "padded": 0.2, "pad": 0},
        # three teachers, an odd vocabulary, rows that start anywhere
        {"name": "step_100x50001_f32_three", "op": "step", "rows": 100, "vocab": 50001, "dtype": "f32", "lists": 3, "k": 17, "temperature": 1.5, "whole": True, "backward": True, "padded": 0.05, "pad": 2},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["sample", "sample", "top", "loss", "step"])
    vocab = _spread(rng, 1000, 256000)
    most = {"sample": 16_000_000, "top": 65_000_000, "loss": 120_000_000, "step": 120_000_000}[op]
    rows = _spread(rng, 1, max(1, min(1024, most // vocab)))
    case = {"op": op, "rows": rows, "vocab": vocab, "dtype": rng.choice(["f32", "bf16", "f16"]), "pad": rng.choice([0, 0, 1, 8, 13])}
    if op == "sample":
        mixed = rng.random() < 0.3
        case.update(law=rng.choice(["gauss", "zipf"]), temperature=round(rng.uniform(0.3, 1.5), 2), top_k=rng.choice([0, _spread(rng, 1, 2000)]), top_p=rng.choice([1.0, round(rng.uniform(0.3, 0.99), 3)]),
                    min_p=rng.choice([0.0, round(rng.uniform(0.001, 0.3), 4)]), mixed=mixed, filtered=rng.random() < 0.5, ruled_out=rng.choice([0.0, 0.0, round(rng.uniform(0.0, 0.99), 2)]))
    elif op == "top":
        case.update(law=rng.choice(["gauss", "zipf"]), k=min(vocab, _spread(rng, 1, 512)), temperature=round(rng.uniform(0.5, 3.0), 2), ruled_out=rng.choice([0.0, round(rng.uniform(0.0, 0.9), 2)]))
    else:
        case.update(lists=rng.choice([1, 1, 2, 4]), k=min(vocab, _spread(rng, 1, 128)), temperature=round(rng.uniform(0.5, 3.0), 2), whole=rng.random() < 0.5, backward=op == "step" or rng.random() < 0.8,
                    padded=rng.choice([0.0, round(rng.uniform(0.0, 0.5), 2)]))
    return case


# ---------------------------------------------------------------------------------------------------------------------
# inputs


def _logits(gen, law, shape):
    """fp32 logits: "gauss" has a broad head, "zipf" the few likely tokens and the long tail of a language model's."""
    if law == "gauss":
        return 2.5 * torch.randn(shape, generator=gen, device="cuda")
    rank = torch.randperm(shape[-1], generator=gen, device="cuda").float() + 1.0
    gumbel = -torch.log(torch.empty(shape, device="cuda").exponential_(1.0, generator=gen))
    return 3.0 * gumbel - 1.1 * torch.log(rank)


def _stored(x, case):
    """In the case's type, with `pad` entries behind each row: a row stride that is not the vocabulary's size."""
    rows, vocab = x.shape
    buf = torch.zeros((rows, vocab + case["pad"]), dtype=_TYPES[case["dtype"]], device="cuda")
    buf[:, :vocab] = x
    return buf[:, :vocab]


def _draws(case, seed):
    """The temperature, k, p and minimum of each row, on the host, as the 32-bit values they are passed in."""
    g = np.random.Generator(np.random.PCG64(seed * 2 + 1))
    n = case["rows"]
    if not case["mixed"]:
        return (np.full(n, case["temperature"], np.float32), np.full(n, case["top_k"], np.int32), np.full(n, case["top_p"], np.float32), np.full(n, case["min_p"], np.float32))
    pick = lambda share, a, b: np.where(g.random(n) < share, a, b)  # noqa: E731
    return (pick(0.1, 0.0, g.uniform(0.5, 1.3, n)).astype(np.float32), pick(0.4, 0, g.integers(1, 400, n)).astype(np.int32),
            pick(0.4, 1.0, g.uniform(0.5, 0.99, n)).astype(np.float32), pick(0.7, 0.0, g.uniform(0.01, 0.2, n)).astype(np.float32))


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    rows, vocab = case["rows"], case["vocab"]
    if case["op"] in ("sample", "top"):
        x = _logits(gen, case["law"], (rows, vocab))
        if case["ruled_out"] > 0.0:
            x.masked_fill_(torch.rand((rows, vocab), generator=gen, device="cuda") < case["ruled_out"], -math.inf)
        state = {"case": case, "logits": _stored(x, case)}
        if case["op"] == "sample":
            state["uniforms"] = torch.rand(rows, generator=gen, device="cuda")
            state["of_rows"] = [torch.from_numpy(v).cuda() for v in _draws(case, seed)]
        return state
    # a student and its teachers, which agree in part; the teachers' lists in the order of their logits
    shared = 2.2 * torch.randn((rows, vocab), generator=gen, device="cuda")
    student = _stored(shared + 1.2 * torch.randn((rows, vocab), generator=gen, device="cuda"), case).detach()
    ids, values, lse = [], [], []
    for _ in range(case["lists"]):
        teacher = shared + 1.2 * torch.randn((rows, vocab), generator=gen, device="cuda")
        v, i = torch.topk(teacher, case["k"], dim=1)
        ids.append(i.int())
        values.append(v)
        lse.append(torch.logsumexp(teacher.double() / case["temperature"], dim=1).float())
    ids, values, lse = torch.stack(ids, 1), torch.stack(values, 1), torch.stack(lse, 1)
    padded = torch.rand(rows, generator=gen, device="cuda") < case["padded"]
    ids[padded] = -1
    weights = (np.arange(case["lists"], 0, -1) / np.arange(1, case["lists"] + 1).sum()).astype(np.float32)
    state = {"case": case, "student": student, "ids": ids.contiguous(), "values": values.contiguous(), "lse": lse.contiguous() if case["whole"] else None, "weights": [float(w) for w in weights]}
    # what the loss of a row counts: an average over the rows in earnest, a few of them weighted down
    state["row_weights"] = (0.5 + torch.rand(rows, generator=gen, device="cuda")) / rows
    if case["op"] == "loss" and case["backward"]:
        state["student"].requires_grad_(True)
    return state


# ---------------------------------------------------------------------------------------------------------------------
# the operators


def _sample(logits, uniforms, temperature, top_k, top_p, min_p, filtered):
    """64 bits throughout: a token is the neighbour of a border of the cumulative sums."""
    rows, vocab = logits.shape
    t, p, least = temperature.double()[:, None], top_p.double()[:, None], min_p.double()[:, None]
    k = torch.where(top_k > 0, top_k, vocab)[:, None]
    v, order = torch.sort(logits.float(), dim=1, descending=True, stable=True)   # equal ones: the lowest index first
    rank = torch.arange(vocab, device=logits.device)[None, :]
    v = v.double()
    z = v - v[:, :1]
    greedy = t == 0.0
    w = torch.where(greedy, (rank == 0).double(), torch.exp(z / torch.where(greedy, 1.0, t)))
    keep = (rank < k) & (v > -math.inf) & ((rank == 0) | ~greedy)
    w = torch.where(keep, w, 0.0)
    run_up = torch.cumsum(w, 1)
    total = run_up[:, -1:]
    keep = keep & ((p >= 1.0) | (run_up - w < p * total)) & (w >= least)
    w = torch.where(keep, w, 0.0)
    kept = torch.zeros_like(keep).scatter_(1, order, keep)
    mass = torch.zeros_like(w).scatter_(1, order, w)
    run_up = torch.cumsum(mass, 1)
    total = run_up[:, -1:]
    reached = (run_up >= uniforms.double()[:, None] * total) & (mass > 0.0)
    token = reached.int().argmax(1)
    out = {"tokens": token.int(), "prob": (mass.gather(1, token[:, None]) / total)[:, 0].float(), "kept": kept.sum(1).int()}
    if filtered:
        out["filtered"] = torch.where(kept, logits, -math.inf)
    return out


def _top(logits, k, temperature):
    x = logits.float()
    v, order = torch.sort(x, dim=1, descending=True, stable=True)
    v, order = v[:, :k], order[:, :k]
    z = x / temperature
    m = z.max(1, keepdim=True).values
    lse = (m + torch.log(torch.exp(z - m).sum(1, keepdim=True)))[:, 0]
    return {"values": v.contiguous(), "ids": torch.where(v > -math.inf, order, -1).int(), "lse": lse}


def _distill(student, ids, values, lse, weights, temperature, row_weights):
    """Loss, and the gradient of its sum weighted by `row_weights` (None: no gradient)."""
    rows, vocab = student.shape
    there = ids >= 0
    v = torch.where(there, values, -math.inf) / temperature
    if lse is None:
        m = torch.clamp(v.max(2, keepdim=True).values, min=-1e30)
        e = torch.exp(v - m)
        t = e / torch.clamp(e.sum(2, keepdim=True), min=1e-30)
    else:
        t = torch.exp(v - lse[:, :, None])
    t = t * torch.tensor(weights, device=t.device)[None, :, None]
    target = torch.zeros((rows, vocab), device=t.device)
    target.scatter_add_(1, torch.where(there, ids, 0).reshape(rows, -1).long(), torch.where(there, t, 0.0).reshape(rows, -1))
    z = student.float() / temperature
    z = z - z.max(1, keepdim=True).values
    log_q = z - torch.log(torch.exp(z).sum(1, keepdim=True))
    loss = torch.where(target > 0.0, target * (torch.log(torch.where(target > 0.0, target, 1.0)) - log_q), 0.0).sum(1)
    if row_weights is None:
        return loss, None
    grad = (row_weights / temperature)[:, None] * (target.sum(1, keepdim=True) * torch.exp(log_q) - target)
    return loss, grad.to(student.dtype)


def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        import paper_2502_01662_b200 as pkg
        if op == "sample":
            if case["mixed"]:
                temperature, top_k, top_p, min_p = state["of_rows"]
            else:
                temperature, top_k, top_p, min_p = case["temperature"], case["top_k"], case["top_p"], case["min_p"]
            got = pkg.sample(state["logits"], state["uniforms"], temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p, filtered=case["filtered"])
            return {k: got[k] for k in ("tokens", "prob", "kept", "filtered") if k in got}
        if op == "top":
            got = pkg.top_logits(state["logits"], case["k"], temperature=case["temperature"])
            return {k: got[k] for k in ("values", "ids", "lse")}
        teacher = (state["ids"], state["values"])
        more = {"lse": state["lse"], "weights": state["weights"], "temperature": case["temperature"]}
        if op == "step":
            got = pkg.distill_step(state["student"], *teacher, row_weights=state["row_weights"], **more)
            return {"loss": got["loss"], "grad": got["grad"]}
        loss = pkg.distill_loss(state["student"], *teacher, **more)
        if not case["backward"]:
            return {"loss": loss}
        grad, = torch.autograd.grad(loss, state["student"], state["row_weights"])
        return {"loss": loss.detach(), "grad": grad}
    if op == "sample":
        return _sample(state["logits"], state["uniforms"], *state["of_rows"], case["filtered"])
    if op == "top":
        return _top(state["logits"], case["k"], case["temperature"])
    loss, grad = _distill(state["student"].detach(), state["ids"], state["values"], state["lse"], state["weights"], case["temperature"], state["row_weights"] if case["backward"] else None)
    return {"loss": loss, "grad": grad} if case["backward"] else {"loss": loss}


def work(case):
    tokens, size = case["rows"] * case["vocab"], _BYTES[case["dtype"]]
    if case["op"] == "sample":
        return {"bytes": tokens * size * (2 if case["filtered"] else 1) + 32 * case["rows"], "flops": 4 * tokens}
    if case["op"] == "top":
        return {"bytes": tokens * size + case["rows"] * (8 * case["k"] + 4), "flops": 4 * tokens}
    entries = case["rows"] * case["lists"] * case["k"]
    return {"bytes": tokens * size * (2 if case["backward"] else 1) + 8 * entries + 8 * case["rows"], "flops": (8 if case["backward"] else 4) * tokens}


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits, row by row


def _exact_sample_row(x, u, t, k, p, least):
    """x: a row in 64 bits (numpy).  The kept tokens in order of (logit down, index up), then the draw in order of the index."""
    order = np.lexsort((np.arange(x.size), -x))
    order = order[x[order] > -np.inf]
    if t == 0.0:
        order = order[:1]
        w = np.ones(1)
    else:
        w = np.exp((x[order] - x[order[0]]) / t)
    if k > 0:
        order, w = order[:k], w[:k]
    if p < 1.0:
        before = np.concatenate(([0.0], np.cumsum(w)[:-1]))
        n = int(np.count_nonzero(before < p * w.sum()))
        order, w = order[:n], w[:n]
    n = int(np.count_nonzero(w >= least))
    order, w = order[:n], w[:n]
    by_index = np.argsort(order)
    cdf = np.cumsum(w[by_index])
    at = min(int(np.searchsorted(cdf, u * cdf[-1], side="left")), n - 1)
    return int(order[by_index][at]), float(w[by_index][at] / cdf[-1]), order


def exact(case, seed):
    state = prepare(case, seed)
    rows, vocab = case["rows"], case["vocab"]
    if case["op"] == "sample":
        x, u = state["logits"].double().cpu().numpy(), state["uniforms"].double().cpu().numpy()
        of = [v.astype(np.float64) for v in _draws(case, seed)]
        tokens, prob, kept, law = np.zeros(rows, np.int32), np.zeros(rows), np.zeros(rows, np.int32), np.full((rows, vocab), -np.inf)
        for r in range(rows):
            tokens[r], prob[r], order = _exact_sample_row(x[r], u[r], of[0][r], int(of[1][r]), of[2][r], of[3][r])
            kept[r] = order.size
            law[r, order] = x[r, order]
        out = {"tokens": tokens, "prob": prob, "kept": kept}
        if case["filtered"]:
            out["filtered"] = law
        return out
    if case["op"] == "top":
        values, ids, lse = [], [], []
        for r in range(rows):
            x = state["logits"][r].double().cpu().numpy()
            order = np.lexsort((np.arange(vocab), -x))[: case["k"]]
            z = x / case["temperature"]
            lse.append(float(z.max() + math.log(float(np.exp(z - z.max()).sum()))))
            values.append(x[order])
            ids.append(np.where(x[order] > -np.inf, order, -1).astype(np.int32))
        return {"values": np.stack(values), "ids": np.stack(ids), "lse": np.array(lse)}
    losses, grads = [], []
    temperature = case["temperature"]
    for lo in range(0, rows, 32):
        part = slice(lo, min(rows, lo + 32))
        s = state["student"].detach()[part].double().requires_grad_(case["backward"])
        log_q = torch.log_softmax(s / temperature, 1)
        mixed = torch.zeros(s.shape, dtype=torch.float64, device="cuda")
        for j in range(case["lists"]):
            for_ids = state["ids"][part, j].long()
            there = (for_ids >= 0).double()
            v = state["values"][part, j].double() / temperature
            share = torch.softmax(v, 1) if state["lse"] is None else torch.exp(v - state["lse"][part, j].double()[:, None])
            mixed.scatter_add_(1, for_ids.clamp(min=0), there * share * float(np.float32(state["weights"][j])))
        loss = torch.xlogy(mixed, mixed).sum(1) - (mixed * log_q).sum(1)
        losses.append(loss.detach())
        if case["backward"]:
            grads.append(torch.autograd.grad((loss * state["row_weights"][part].double()).sum(), s)[0])
    out = {"loss": torch.cat(losses)}
    if case["backward"]:
        out["grad"] = torch.cat(grads)
    return out
