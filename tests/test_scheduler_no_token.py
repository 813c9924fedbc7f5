"""A model whose logits hold no distribution ends a run with an error; its tokens are not -1."""
import numpy as np
import pytest

from oracle import cos_oracle as orc
from paper_2502_01662_b200 import scheduler as sch

from test_scheduler import oracle_verify, oracle_verify_n

WE, V = orc.COMBINE_PROB_ENSEMBLE, 40


class Nothing:
    """A proposer as the library's is where a row holds a NaN."""
    temperature = 0.9

    def draw(self, row, uniform):
        return -1 if np.isnan(row).any() else 3

    def law(self, rows):
        return rows


def models(n, bad):
    out = sch.make_table_models(n, V, contexts=16, seed=8)
    for i in bad:
        out[i].table[5:] = np.nan
    return out


@pytest.mark.parametrize("bad", [[0], [1], [0, 1]])
@pytest.mark.parametrize("propose", [None, Nothing()])
def test_no_distribution(bad, propose):
    for run in (sch.AlternateProposal(models(2, bad), (3, 2), 0.9, oracle_verify(WE, (0.5, 0.5), 0.9, V), propose=propose),
                sch.CollaborativeSpeculation(models(3, bad), (2, 2, 1), 0.9, oracle_verify_n(3, WE, (0.5, 0.3, 0.2), 0.9, V), propose=propose)):
        with np.errstate(invalid="ignore"), pytest.raises(ValueError, match="no token"):
            run.generate([1], 400)


def test_runs_without_any_stay():
    for propose in (None, Nothing()):
        tokens, _ = sch.AlternateProposal(models(2, []), (3, 2), 0.9, oracle_verify(WE, (0.5, 0.5), 0.9, V), propose=propose).generate([1], 60)
        assert min(tokens) >= 0
