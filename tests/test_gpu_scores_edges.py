"""Edges of the modified scores: masked pairs whose scores overflow, rows that a short tile leaves in LDS, slopes at the
ends of their range.

The cap takes a shorter polynomial where all scores of a block are small.  A masked pair's score may be NaN (finite
values whose products overflow to both infinities) and must not hide a score of its block that is beyond the
polynomial's range, nor reach a gradient.  Rows past a short tile's end must not count either: before each of those
cases the kernels run on full tiles of one value in every CU's LDS, NaN among them, and results are right, and the same
bits whatever LDS held."""
import math

import numpy as np
import pytest
import torch

from paper_2609_34318_amd import hydra, ring

from test_gpu_scores import BF16, MODS, Setup, _check_forward, _check_grads

pytestmark = pytest.mark.gpu


def _overflowing(which, mod):
    """Blocks of 16 rows of one document and 16 of the next, in turn: the products of the one's keys (or queries) with the
    other's rows overflow to infinities of both signs.  The one's own scores are 0, and so are its values and
    gradients."""
    docs = [16, 16] * 6 + [48, 48]
    n = sum(docs)
    s = Setup((docs, 2, 1, [(0, n)], [[(0, n)]]), mod, seed=11)
    k, v = s.kv[0]
    huge = torch.where(torch.arange(192, device="cuda") % 2 == 0, 3e38, -3e38).to(BF16)
    ones = torch.from_numpy(np.repeat([i % 2 == 0 for i in range(len(docs))], docs)).cuda()
    big, zero = (k, s.q) if which == "keys" else (s.q, k)
    big[ones], zero[ones], v[ones], s.do[ones] = huge, 0, 0, 0
    assert bool(torch.isnan(zero[~ones].float() @ huge.float()).any())
    return s


@pytest.mark.parametrize("mod", MODS)
@pytest.mark.parametrize("which", ["keys", "queries"])
def test_masked_scores_that_overflow(which, mod):
    s = _overflowing(which, mod)
    O, L, _, _ = s.reference()
    sh = s.share()
    ring.forward(sh, s.q, s.kv)
    torch.cuda.synchronize()
    _check_forward(s, sh, O, L, which)


@pytest.mark.parametrize("ds", [False, True])
@pytest.mark.parametrize("mod", MODS)
@pytest.mark.parametrize("which", ["keys", "queries"])
def test_gradients_beside_masked_scores_that_overflow(which, mod, ds):
    s = _overflowing(which, mod)
    _, _, rq, rkv = s.reference()
    sh = s.share(ds)
    assert (sh.ds_buf is not None) == ds
    ring.forward(sh, s.q, s.kv)
    dq, dkv = s.grads()
    ring.backward(sh, s.q, s.kv, s.do, dq, dkv)
    torch.cuda.synchronize()
    _check_grads((dq, dkv), (rq, rkv), which)


def _poison(value):
    """Forward and both backwards over 512 rows x 256 heads of `value`, more workgroups than CUs."""
    n, H = 512, 256
    full = lambda d: torch.full((n, H, d), value, dtype=BF16, device="cuda")  # noqa: E731
    sh = ring.make_share([0, n], H, [(0, n)], [[(0, n)]], ds_kv_heads=H, scores=hydra.Scores(50.0))
    q, k, v, do = full(192), full(192), full(128), full(128)
    ring.forward(sh, q, [(k, v)])
    p, (dq, dk, dv) = sh.problems[0], (torch.zeros((n, H, d), device="cuda") for d in (192, 192, 128))
    hydra.attn_bwd_ds(p, q, k, v, sh.o_acc, sh.lse_acc, do, dq, dk, dv, sh.ds_buf, sh.workspace)
    hydra.attn_bwd(p, q, k, v, sh.o_acc, sh.lse_acc, do, dq, dk, dv, sh.workspace)


def _run(s, sh, value):
    for t in (sh.o_acc, sh.lse_acc, sh.o_bf16):
        t.fill_(math.nan)
    _poison(value)
    ring.forward(sh, s.q, s.kv)
    dq, dkv = s.grads()
    _poison(value)
    ring.backward(sh, s.q, s.kv, s.do, dq, dkv)
    torch.cuda.synchronize()
    return dq, dkv


ROWS = {f"whole_{n}": ([n], 2, 1, [(0, n)], [[(0, n)]]) for n in (1, 5, 23, 31, 32, 33, 40, 63, 96, 131)}
ROWS.update({f"last_row_of_{n}": ([n], 2, 2, [(n - 1, 1)], [[(0, n)]]) for n in (65, 70, 87, 96, 127, 160)})
ROWS["short_chunks"] = ([30, 70, 3], 2, 1, [(0, 103)], [[(0, 7)], [(7, 20), (40, 9)], [(27, 13), (49, 54)]])


@pytest.mark.parametrize("mod", MODS)
@pytest.mark.parametrize("case", ROWS)
def test_rows_left_in_lds(case, mod):
    s = Setup(ROWS[case], mod, seed=7)
    O, L, rq, rkv = s.reference()
    for ds in (False, True):
        sh = s.share(ds)
        if ds and sh.ds_buf is None:
            continue
        first = None
        for value in (math.nan, 0.0, 300.0):
            dq, dkv = _run(s, sh, value)
            _check_forward(s, sh, O, L, (case, ds, value))
            _check_grads((dq, dkv), (rq, rkv), (case, ds, value))
            out = [t.clone() for t in (sh.o_acc, sh.lse_acc, sh.o_bf16, dq, *[x for p in dkv for x in p])]
            if first is None:
                first = out
            assert all(torch.equal(a, b) for a, b in zip(first, out)), (ds, value)


def test_slopes_at_the_ends_of_their_range():
    """Slopes whose multiple of log2(e) is beyond 32 bits: a row's own key, at distance 0, is all it sees, and the next
    one where the head's slope is 0."""
    n, most = 70, torch.finfo(torch.float32).max
    for mod in ("bias", "all_no_prefix"):
        s = Setup(([n], 3, 1, [(0, n)], [[(0, n)]]), mod, seed=13)
        s.slopes.copy_(torch.tensor([most, 2.4e38, 0.0]))
        O, L, rq, rkv = s.reference()
        sh = s.share()
        ring.forward(sh, s.q, s.kv)
        _check_forward(s, sh, O, L, mod)
        dq, dkv = s.grads()
        ring.backward(sh, s.q, s.kv, s.do, dq, dkv)
        torch.cuda.synchronize()
        assert torch.equal(sh.o_acc[:, :2], s.kv[0][1].float().expand(-1, 2, -1))
        _check_grads((dq, dkv), (rq, rkv), mod)
