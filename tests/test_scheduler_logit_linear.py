"""Schedulers that combine logits take no proposer that rules tokens out: the combination would not be a number there, and the run's tokens none."""
import pytest

from oracle import cos_oracle as orc
from paper_2502_01662_b200 import scheduler as sch

from test_scheduler import oracle_verify
from test_scheduler_propose import NumpyProposer

LL, WE = orc.COMBINE_LOGIT_LINEAR, orc.COMBINE_PROB_ENSEMBLE
V = 50


def runs(verify, verify_n, T, propose):
    """Both schedulers, as they are made."""
    yield lambda: sch.AlternateProposal(sch.make_table_models(2, V, contexts=16, seed=5), (3, 2), T, verify, propose=propose)
    yield lambda: sch.CollaborativeSpeculation(sch.make_table_models(3, V, contexts=16, seed=5), (3, 2, 1), T, verify_n, propose=propose)


@pytest.mark.parametrize("T,limits,refused", [(0.9, dict(top_k=4), True), (0.9, dict(top_p=0.9), True), (0.9, dict(min_p=0.1), True), (0.0, {}, True), (0.0, dict(top_k=4), True),
                                              (0.9, {}, False), (0.9, dict(top_k=V), False), (0.9, dict(top_k=-1), False)])
def test_what_a_logit_linear_run_takes(T, limits, refused):
    propose = sch.GpuProposer(T, **limits)
    assert propose.rules_out(V) == refused
    for combine in (LL, WE):
        two, three = sch.gpu_verify(combine, (0.5, 0.5), T, V), sch.gpu_verify(combine, (0.5, 0.3, 0.2), T, V)
        for make in runs(two, three, T, propose):
            if refused and combine == LL:
                with pytest.raises(ValueError, match="logit-linear"):
                    make()
            else:
                make()
        for make in runs(two, three, T, None):
            make()
        for make in runs(two, three, T + 1.0, propose):
            with pytest.raises(ValueError, match="temperature"):
                make()


def test_proposers_and_verifications_that_say_nothing():
    """... are taken at their word, as before; one without limits draws the tokens of a run without a proposer."""
    T, out = 0.9, []
    for propose in (None, NumpyProposer(T)):
        verify = oracle_verify(LL, (1.5, -0.5), T, V)
        verify.logit_linear = True
        run = sch.AlternateProposal(sch.make_table_models(2, V, contexts=16, seed=5), (3, 2), T, verify, propose=propose)
        out.append(run.generate([0], 40)[0])
    assert out[0] == out[1] and min(out[0]) >= 0
