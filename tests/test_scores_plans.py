"""What the plan and the workspace of modified scores depend on (hydra_scores.h): the prefixes, and whether the scores are
modified at all; not the cap or the slopes.  (Planned calls on plans of other scores: test_gpu_scores.py.)"""
import numpy as np
import pytest

from paper_2609_34318_amd import hydra

CU = list(range(0, 601))  # as many documents as tokens: their prefix ends need room of their own
SEG = [(0, 600)]


def _problem(cap=0.0, slopes=False, prefix=None):
    sc = hydra.Scores(cap, None, prefix)
    if slopes:
        sc.c.slopes = 1 << 20  # an address that the host does not read
    return hydra.Problem(CU, 2, SEG, SEG, scores=sc)


@pytest.mark.parametrize("kw", [dict(cap=5.0), dict(slopes=True), dict(prefix=[0] * 600), dict(cap=30.0, slopes=True),
                                dict(cap=5.0, prefix=[0] * 600)])
def test_one_plan_for_cap_and_slopes(kw):
    a, b = _problem(cap=30.0), _problem(**kw)
    assert hydra.workspace_size(a) == hydra.workspace_size(b)
    for which in (0, 1):
        assert np.array_equal(hydra.plan_items(a, which), hydra.plan_items(b, which))


def test_unmodified_scores_have_another_workspace():
    none = _problem()
    assert hydra.workspace_size(none) == hydra.lib().hydra_workspace_size(none.ref)
    assert hydra.workspace_size(none) < hydra.workspace_size(_problem(cap=30.0))
