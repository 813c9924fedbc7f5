"""The proposer's operators in 64 bits (numpy), row by row from their definitions, and the tolerances they are held to.

Sampling.  The library sums weights as whole multiples of a unit of 2^-scale of the largest one, scale = min(46, 63 - ceil(log2 V)); each is off by half a
unit and by the error of its evaluation (below 2^-44 of it; weights below 2^-36 by 2^-17 of them, at most 2^-53), so no sum is off by more than
`slack` = V (unit / 2 + 2^-53) + S 2^-43, in units of the largest weight.  `check_sample` wants every border (of top-p, of the draw) on the right side of its threshold up to that, and everything else exact."""
import math

import numpy as np
import torch

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def check_sample(x, u, T, k, p, least, token, prob, kept, status, law=None):
    """x: one row in float64; token, prob, kept, status: what came back for it; law: its filtered logits in float64."""
    V = x.size
    if not np.all(x < np.inf) or np.all(x == -np.inf) or not T >= 0:      # (NaN fails the first comparison)
        assert (token, kept, status) == (-1, 0, 1) and math.isnan(prob), (token, kept, status, prob)
        if law is not None:
            assert np.array_equal(law, x, equal_nan=True)
        return
    assert status == 0
    x = x + 0.0
    line = np.lexsort((np.arange(V), -x))
    line = line[x[line] > -np.inf]
    if T == 0.0:
        assert (token, prob, kept) == (line[0], 1.0, 1)
        want = line[:1]
    else:
        with np.errstate(under="ignore"):
            w = np.exp((x[line] - x[line[0]]) / T)
        slack = V * (2.0 ** -(min(46, 63 - math.ceil(math.log2(V))) + 1) + 2.0 ** -53) + w.sum() * 2.0 ** -43
        n = line.size if k <= 0 else min(k, line.size)
        if p < 1.0:
            before = np.concatenate(([0.0], np.cumsum(w[:n])))
            target = max(p, 0.0) * before[n]
            sure = int(np.count_nonzero(before[:n] < target - 2 * slack))
            possible = max(1, int(np.count_nonzero(before[:n] < target + 2 * slack)))
        else:
            sure = possible = n
        lo = int(np.count_nonzero(w[:sure] >= least * (1 + 2.0 ** -40)))
        hi = int(np.count_nonzero(w[:possible] >= least * (1 - 2.0 ** -40)))
        assert max(lo, 1) <= kept <= max(hi, 1), (lo, kept, hi)
        want, w = line[:kept], w[:kept]
        up = np.argsort(want)
        cdf = np.cumsum(w[up])
        u = min(max(u, 0.0), 1.0) if u == u else 0.0
        at = np.searchsorted(want[up], token)
        assert at < kept and want[up][at] == token, (token, kept)
        target = u * cdf[-1]
        assert cdf[at] >= target - 2 * slack and (cdf[at - 1] if at else 0.0) <= target + 2 * slack, (token, target, cdf[max(at - 1, 0):at + 1])
        true = w[up][at] / cdf[-1]
        assert abs(prob - true) <= true * (2.0 ** -24 + 2.0 ** -40 + 2 * slack / cdf[-1]) + 2.0 ** -149, (prob, true)
    if law is not None:
        expect = np.full(V, -np.inf)
        expect[want] = x[want]
        assert np.array_equal(law, expect)


def check_samples(logits, u, T, k, p, least, out):
    """A whole call: T, k, p, least as numbers or arrays of the rows."""
    x = logits.double().cpu().numpy()
    rows = x.shape[0]
    of = [np.broadcast_to(np.asarray(v, dtype), (rows,)) for v, dtype in ((T, np.float32), (k, np.int64), (p, np.float32), (least, np.float32))]
    got = {name: v.double().cpu().numpy() for name, v in out.items()}
    u = u.double().cpu().numpy()
    for r in range(rows):
        m = float(of[3][r])
        check_sample(x[r], u[r], float(of[0][r]), int(of[1][r]), float(of[2][r]), min(max(m, 0.0), 1.0), int(got["tokens"][r]), float(got["prob"][r]), int(got["kept"][r]),
                     int(got["row_status"][r]), got["filtered"][r] if "filtered" in got else None)


# Log-sum-exp.  A term 2^-a of the largest is exp2 of a product of rounded factors: 3 roundings of the argument, a 3 2^-24 ln 2 < a 1.1 2^-23, and 2^-22 of the
# exponential; weighted by their shares the a average to at most log2 V.  Eight terms are added in 32 bits (7 2^-24).  A running maximum that moves multiplies what
# is there by another exponential (2^-22 each; on random data a lane sees a new maximum less than 16 times).
def lse_error(V):
    return 17 * 2.0 ** -22 + 7 * 2.0 ** -24 + 1.1 * 2.0 ** -23 * math.log2(max(V, 2))


def top_of(x, k, T):
    """values, ids, lse of one row (float64)."""
    if not np.all(x < np.inf):
        return np.full(k, -np.inf), np.full(k, -1), math.nan
    line = np.lexsort((np.arange(x.size), -(x + 0.0)))[:k]
    v = x[line]
    m = x.max()
    lse = -math.inf if m == -np.inf else m / T + math.log(np.exp((x - m) / T).sum())
    return v, np.where(v > -np.inf, line, -1), lse


def distill(s, ids, values, lse, weights, T):
    """loss, gradient of the loss, target, q of one row: s [V] float64, ids and values [lists, k], lse [lists] or None."""
    V = s.size
    t = np.zeros(V)
    for g in range(ids.shape[0]):
        there = (ids[g] >= 0) & (values[g] > -np.inf)
        if not there.any():
            continue
        v = values[g][there] / T
        share = np.exp(v - lse[g]) if lse is not None else np.exp(v - v.max()) / np.exp(v - v.max()).sum()
        np.add.at(t, ids[g][there], float(np.float32(weights[g])) * share)
    if not t.any():
        return 0.0, np.zeros(V), t, np.zeros(V)
    z = s / T
    m = z.max()
    log_z = m + math.log(np.exp(z - m).sum())
    with np.errstate(divide="ignore"):
        log_q = z - log_z
    at = t > 0
    loss = float(np.sum(t[at] * (np.log(t[at]) - log_q[at])))
    q = np.exp(log_q)
    return loss, (t.sum() * q - t) / T, t, q


def check_loss(got, want, t, V, extra=0.0):
    if not math.isfinite(want):
        assert got == want, (got, want)
        return
    assert abs(got - want) <= t.sum() * (lse_error(V) + 2.0 ** -22) + abs(want) * 2.0 ** -24 + 2.0 ** -126 + extra, (got, want)


def check_grad(got, want, q, t, s, T, weight, dtype):
    """Gradient of weight * loss, against `want` times the weight."""
    V = s.size
    with np.errstate(divide="ignore", invalid="ignore"):
        a = np.where(s > -np.inf, (s.max() - s) / T, 0.0) / math.log(2.0)
    log_z = np.log2(1.0 / q.max()) if q.max() > 0 else 0.0
    # of q: the normaliser, its logarithm as a 32-bit number, the argument and the exponential; three roundings of the factors in front; all of 32 bits
    rel = lse_error(V) + 2.0 ** -22 + 1.1 * 2.0 ** -23 * (a + log_z) + 3 * 2.0 ** -24
    info = torch.finfo(dtype)
    tol = abs(weight) * t.sum() / T * q * rel + np.abs(want * weight) * (info.eps / 2 + 2.0 ** -24) + info.smallest_normal * info.eps + 2.0 ** -126
    assert np.all(np.abs(got - want * weight) <= tol), float(np.max(np.abs(got - want * weight) / tol))
