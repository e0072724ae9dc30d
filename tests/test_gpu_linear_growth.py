"""Linear attention whose decays grow: every product of e^(g d) that the definition has fits 32 bits, the ones of rows
that do not exist would not.

Tolerances: those of test_gpu_linear.py, but for the weights.  e^x of x = g d has there a term's own e^-x to spare;
here it counts in full: log2(e) and its products by g and by d are rounded once each, so that e^x is off by
3 |x| 2^-24 of itself, x up to g n over a sequence of n rows.
"""
import numpy as np
import pytest
import torch

from paper_2609_34318_amd import hydra
from test_gpu_linear import cuda, draw, np64, reference, run

pytestmark = pytest.mark.gpu


def check(cu, x, got):
    want, size = reference(cu, x), reference(cu, x, absolute=True)
    rows = max(np.diff(cu).max(), 1)
    grown = 3 * float(x["decay"].max()) * rows * 2.0 ** -24
    for n, t in got.items():
        t = np64(t)
        if n in ("state", "d_state"):
            tol = size[n] * (3 * rows * 2.0 ** -24 + (rows // 32 + 2) * 2.0 ** -22 + grown) + 1e-30
        else:
            assert (t[cu[-1]:] == 7.0).all(), n
            t = t[:cu[-1]]
            tol = np.abs(want[n]) * 2.0 ** -8 + size[n] * (2.0 ** -14 + (0 if n == "o" else 2.0 ** -8) + 3 * rows * 2.0 ** -24 + grown) + 1e-30
        assert np.isfinite(want[n]).all() and np.abs(want[n]).max() < 2.0 ** 126  # the definition fits 32 bits
        bad = ~np.isfinite(t)
        assert not bad.any(), (n, int(bad.sum()), np.argwhere(bad)[0])
        assert (np.abs(t - want[n]) / tol).max(initial=0.0) <= 1, (n, (np.abs(t - want[n]) / tol).max())


CASES = [  # rows of each sequence, log decays, K/V heads
    ([5, 20, 27, 1, 12], [1.0, 3.0], 2),    # one chunk, rows that are not there at e^93
    ([31, 5, 30, 13], [1.0, 2.5], 1),
    ([1, 1], [80.0, 3.0], 2),
    ([33, 40, 80, 64], [1.0, 0.5], 2),      # a chunk of a few rows, then whole ones
    ([50, 2, 29], [0.01, 1.5], 1),
    ([300, 129, 7], [0.25, -0.5], 2),       # cut into items of 128 rows
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[0] + c[1])))
@pytest.mark.parametrize("dims", [(64, 64), (192, 128), (128, 64), (64, 128)], ids=lambda d: f"{d[0]}x{d[1]}")
@pytest.mark.parametrize("states", [True, False], ids=["states", "zero"])
def test_growing_decays(case, dims, states):
    lengths, decay, Hk = case
    cu = np.concatenate([[0], np.cumsum(lengths)])
    x = draw(sum(lengths), cu[-1] + 3, 2, Hk, *dims, len(lengths), states, decay=decay)
    check(cu, x, run(hydra.Linear(cu, 2, *dims, n_kv_heads=Hk), cuda(x)))


def test_growing_decays_of_a_step():
    """One row of zero states: e^80 of nothing."""
    x = cuda(draw(1, 2, 2, 2, 64, 64, 2, decay=[80.0, 3.0]))
    o, state = torch.empty((2, 2, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 2, 64, 64), device="cuda")
    hydra.linear_step(x["q"], x["k"], x["v"], x["decay"], state, o)
    want = x["k"].float()[:, :, :, None] * x["v"].float()[:, :, None]
    assert torch.equal(state, want) and torch.isfinite(o.float()).all()
