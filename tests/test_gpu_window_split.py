"""Windows with sinks in full launches, whose items with the sinks are split all the same, and query tiles whose sinks and
window lie in more segments than a record holds, against the fp64 oracle.

Tolerances: those of test_gpu_window.py, and the same for the rows of the sinks by themselves: their sums have the same
terms, each rounded once to bf16.
"""
import numpy as np
import pytest
import torch

from oracle import scores as S
from paper_2609_34318_amd import hydra
from test_gpu_window import TOL_GRAD, Setup, check

pytestmark = pytest.mark.gpu


def f(t):
    return t.float().cpu().numpy()


FULL = {  # documents, query heads, K/V heads, window, sinks: 512 and more items of 128 keys
    "documents": ([1, 3000, 1223], 16, 16, 200, 4),
    "heads_on_all_cus": ([5632], 12, 12, 64, 130),
    "gqa": ([4224], 32, 16, 40, 9),
}


def full_setup(name):
    docs, H, Hkv, window, sinks = FULL[name]
    T = sum(docs)
    s = Setup((docs, H, Hkv, [(0, T)], [[(0, T)]]), "window")
    s.scores = hydra.Scores(window=window, sinks=sinks)
    return s, dict(window=window, sinks=sinks)


def run_named(s, sh):
    hydra.profile_start()
    got = [t.clone() for t in s.run(sh)]
    return got, hydra.profile_stop()


@pytest.mark.parametrize("name", FULL)
def test_full_launches_split_the_sinks(name):
    """The recompute and the stored-dS backward, split and (without scratch) whole; three K/V heads against the oracle."""
    s, kw = full_setup(name)
    docs, H, Hkv, _, sinks = FULL[name]
    grp, kv_heads = H // Hkv, [0, Hkv // 2 + 1, Hkv - 1]
    heads = [h * grp + i for h in kv_heads for i in range(grp)]
    q, do, (k, v) = f(s.q[:, heads]), f(s.do[:, heads]), [f(t[:, kv_heads]) for t in s.kv[0]]
    O, L = S.attn_fwd(q, k, v, s.cu, s.q_segs, s.steps[0], **kw)
    want = S.attn_bwd(q, k, v, O, L, do, s.cu, s.q_segs, s.steps[0], **kw)
    sink_rows = np.concatenate([np.arange(a, min(a + sinks, b)) for a, b in zip(s.cu[:-1], s.cu[1:])])
    for ds in (False, True):
        whole, names = run_named(s, s.share(ds, scratch=False))
        assert "bwd_merge" not in names
        got, names = run_named(s, s.share(ds))
        assert ("bwd_dkdv_ds_scores" if ds else "bwd_recompute_scores") in names and "bwd_merge" in names  # was split
        o, lse = f(got[0][:, heads]), f(got[1][heads])
        assert np.abs(o - O).max() <= 1.1 * 2.0 ** -8 * float(s.kv[0][1].float().abs().max())
        assert np.abs(lse - L).max() <= 1e-4 + 2.0 ** -21 * np.abs(L).max()
        for i, (x, y) in enumerate(zip((got[3][:, heads], got[4][:, kv_heads], got[5][:, kv_heads]), want)):
            x = f(x)
            assert np.isfinite(x).all()
            for rows in (slice(None), sink_rows):
                assert np.linalg.norm(x[rows] - y[rows]) <= TOL_GRAD * np.linalg.norm(y[rows]) + 2.0 ** -18 * x[rows].size ** 0.5, (ds, i)
        # all heads: the same terms in another order of 32-bit sums, at most one rounding to bf16 of a term apart
        for i, (x, y) in enumerate(zip(got[3:], whole[3:])):
            for rows in (slice(None), sink_rows):
                assert (x[rows] - y[rows]).norm() <= 2.0 ** -8 * y[rows].norm(), (ds, i)
        assert all(torch.equal(a, b) for a, b in zip(got, run_named(s, s.share(ds))[0]))


@pytest.mark.parametrize("kv", [[(0, 100), (150, 100), (300, 3200), (3600, 700)], [(0, 96), (160, 96), (320, 3168), (3584, 704)]],
                         ids=["odd", "aligned"])
def test_more_segments_than_a_record_holds(kv):
    s = Setup(([5000], 2, 1, [(4000, 256)], [kv]), "window")
    s.scores, s.kw = hydra.Scores(window=1000, sinks=350), dict(window=1000, sinks=350)
    want = s.reference()
    p = s.share().problems[0]
    assert hydra.plan_items(p, 0)[0, 3] == 4
    for scratch, ds in ((True, False), (False, False), (True, True)):
        sh = s.share(ds, scratch)
        if ds and sh.ds_buf is None:
            continue
        check(s, s.run(sh), want, (scratch, ds))
