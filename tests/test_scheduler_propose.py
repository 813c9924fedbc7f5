"""The schedulers with a proposer passed in: proposals under top-k, top-p and min-p, here drawn in numpy, verified by the oracle."""
import numpy as np
import pytest
from scipy.special import softmax as sp_softmax
from scipy.stats import chi2 as chi2_dist

from oracle import cos_oracle as orc
from paper_2502_01662_b200 import scheduler as sch

from test_scheduler import oracle_verify, oracle_verify_n

WE = orc.COMBINE_PROB_ENSEMBLE


class NumpyProposer:
    """The methods of GpuProposer, from the definition (float64)."""

    def __init__(self, temperature, top_k=0, top_p=1.0, min_p=0.0):
        self.temperature, self.k, self.p, self.m = float(temperature), top_k, float(np.float32(top_p)), float(np.float32(min_p))

    def _line(self, row):
        x = row.astype(np.float64)
        line = np.lexsort((np.arange(x.size), -x))
        if self.temperature == 0.0:
            return line[:1], np.ones(1)
        w = np.exp((x[line] - x[line[0]]) / float(np.float32(self.temperature)))
        n = min(self.k, x.size) if self.k > 0 else x.size
        if self.p < 1.0:
            n = int(np.count_nonzero(np.concatenate(([0.0], np.cumsum(w[:n])[:-1])) < self.p * w[:n].sum()))
        n = int(np.count_nonzero(w[:n] >= self.m))
        return line[:n], w[:n]

    def draw(self, row, uniform):
        line, w = self._line(row)
        up = np.argsort(line)
        cdf = np.cumsum(w[up])
        return int(line[up][min(int(np.searchsorted(cdf, float(np.float32(uniform)) * cdf[-1])), line.size - 1)])

    def law(self, rows):
        out = np.full_like(rows, -np.inf)
        flat, to = rows.reshape(-1, rows.shape[-1]), out.reshape(-1, rows.shape[-1])
        for a, b in zip(flat, to):
            line = self._line(a)[0]
            b[line] = a[line]
        return out


@pytest.mark.parametrize("limits", [dict(top_k=4), dict(top_p=0.7), dict(min_p=0.2), dict(top_k=8, top_p=0.9, min_p=0.05)])
def test_output_follows_the_combination_of_what_the_limits_leave(limits):
    V, T, N, w = 12, 0.9, 4000, (0.4, 0.6)
    models = sch.make_table_models(2, V, contexts=1, seed=5, sigma=1.2, rho=0.6)
    prop = NumpyProposer(T, **limits)
    run = sch.AlternateProposal(models, (3, 2), T, oracle_verify(WE, w, T, V), propose_seed=11, verify_seed=12, propose=prop)
    tokens, _ = run.generate([0], N)
    w64 = np.asarray(w, np.float32).astype(np.float64)
    r = sum(w64[i] * sp_softmax(prop.law(models[i].table)[0].astype(np.float64) / T) for i in range(2))
    counts = np.bincount(np.asarray(tokens), minlength=V)
    assert counts[r == 0].sum() == 0
    at = r > 0
    stat = float(np.sum((counts[at] - len(tokens) * r[at]) ** 2 / (len(tokens) * r[at])))
    assert chi2_dist.sf(stat, int(at.sum()) - 1) > 1e-4, (stat, counts, len(tokens) * r)


def test_three_models_and_greedy():
    V = 300
    models = sch.make_table_models(3, V, contexts=16, seed=6, sigma=2.0, rho=0.9)
    prop = NumpyProposer(0.8, top_k=20)
    run = sch.CollaborativeSpeculation(models, (2, 2, 1), 0.8, oracle_verify_n(3, WE, (0.5, 0.3, 0.2), 0.8, V), propose=prop)
    tokens, _ = run.generate([1], 60)
    assert len(tokens) >= 60
    # without limits, and greedy: the tokens of a run without a proposer
    for T in (0.0, 0.8):
        def go(propose):
            m = sch.make_table_models(2, V, contexts=16, seed=7, sigma=2.0, rho=0.9)
            return sch.AlternateProposal(m, (3, 2), T, oracle_verify(WE, (0.5, 0.5), T, V), propose=propose).generate([1], 60)[0]
        assert go(NumpyProposer(T)) == go(None)


def test_the_temperature_has_to_be_the_runs():
    models = sch.make_table_models(2, 10, contexts=1, seed=1)
    for run in (sch.AlternateProposal, sch.CollaborativeSpeculation):
        with pytest.raises(ValueError):
            run(models, (2, 2), 1.0, None, propose=NumpyProposer(0.5))
