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

from paper_2609_34318_amd import hydra, placement, ring

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


@pytest.mark.parametrize("ds", [False, True])
def test_visible_scores_that_overflow(ds):
    """Products of finite values that are infinite: the scores are at the cap, of either sign, and do not move."""
    n = 96
    s = Setup(([n], 2, 1, [(0, n)], [[(0, n)]]), "cap")
    s.cap, s.scores = 5.0, hydra.Scores(5.0)
    up = torch.arange(n, device="cuda") % 3 != 0  # queries of one sign, keys of both
    s.q.fill_(1e30)
    s.kv[0][0].copy_(torch.where(up, 1e30, -1e30)[:, None, None].to(BF16).expand(n, 1, 192))
    sh = s.share(ds)
    assert (sh.ds_buf is not None) == ds
    ring.forward(sh, s.q, s.kv)
    score = np.where(up.cpu().numpy(), 5.0, -5.0)
    want = np.array([np.logaddexp.reduce(score[:i + 1]) for i in range(n)])
    assert np.abs(sh.lse_acc.cpu().numpy() - want).max() <= 2.0 ** -18 * 10
    dq, dkv = s.grads()
    ring.backward(sh, s.q, s.kv, s.do, dq, dkv)
    torch.cuda.synchronize()
    assert not dq.any() and not dkv[0][0].any() and bool(torch.isfinite(dkv[0][1]).all())


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

# ------------------------------------------------------------------ how far a score may be off

def _key_scores(q, k, scale, cap, slopes):
    """The score of every row against key 0 of its document, which is its LSE where it sees that key alone; and in 64 bits
    A (the products' magnitudes summed), the capped score and the bias."""
    n, H = q.shape[:2]
    p = hydra.Problem([0, n], H, [(0, n)], [(0, 1)], softmax_scale=scale, n_kv_heads=1,
                      scores=hydra.Scores(cap, slopes, None if cap or slopes is not None else [0]))
    ws = torch.empty(hydra.workspace_size(p), dtype=torch.uint8, device="cuda")
    o, lse = torch.empty((n, H, 128), device="cuda"), torch.empty((H, n), device="cuda")
    hydra.attn_fwd(p, q, k, torch.zeros((1, 1, 128), dtype=BF16, device="cuda"), o, lse, ws)
    torch.cuda.synchronize()
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    tau = float(np.float32(scale))
    terms = f(q) * f(k)[:, 0]
    A, s = tau * np.abs(terms).sum(-1).T, tau * terms.sum(-1).T
    if cap:
        s = cap * np.tanh(s / cap)
    B = np.zeros((H, n)) if slopes is None else f(slopes)[:, None] * np.arange(n)[None]
    return f(lse), A, s, B


@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("cap,scale,size", [(0.0, 192 ** -0.5, 1.0), (0.0, 0.25, 1000.0), (50.0, 192 ** -0.5, 8.0),
                                            (1024.0, 0.25, 60.0), (2.0 ** -10, 0.25, 0.01), (30.0, 1.0, 1.0)])
@pytest.mark.parametrize("columns", [1, 192])
def test_scores_are_as_near_as_stated(columns, cap, scale, size, biased):
    """hydra_scores.h: off by at most 2^-16 A + 2^-21 (|s| + B), with a cap by 2^-19 |s| besides.  192 sums that are off
    by half a step, 2^-24, of at most A: 192 2^-24 < 2^-16 of A; none where all columns but one are 0, whose product is
    exact.  Behind them lie at most seven roundings of s (scale times log2 e and that constant, the product, the bias'
    multiply-add, ln 2 and its product in the LSE, and one to spare) and as many of the bias (slope times log2 e and that
    constant, the distance, the multiply-add, ln 2 and its product): less than 8 2^-24 of each.  tanh: the polynomial's
    6e-7 and seven roundings of 2^-24, less than 2^-19."""
    g = torch.Generator(device="cuda").manual_seed(17)
    n, H = 700, 4
    q = torch.randn((n, H, 192), generator=g, device="cuda") * size
    k = torch.randn((1, 1, 192), generator=g, device="cuda")
    q[..., columns:] = 0
    slopes = torch.tensor([0.5, 0.01, 1e-4, 3.0], device="cuda") if biased else None
    lse, A, s, B = _key_scores(q.to(BF16), k.to(BF16), scale, cap, slopes)
    allowed = 2.0 ** -21 * (np.abs(s) + B) + (2.0 ** -19 * np.abs(s) if cap else 0) + (2.0 ** -16 * A if columns > 1 else 0)
    assert (np.abs(lse - (s - B)) <= allowed).all()


# ------------------------------------------------------------------ what the other tests leave out

@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("cap", [2.0 ** -10, 2.0 ** 10])
def test_caps_at_the_ends_of_their_range(cap, sign):
    """Scores far beyond the cap, and scores around it, at the smallest and the largest cap."""
    n = 130
    s = Setup(([n], 2, 1, [(0, n)], [[(0, n)]]), "cap", seed=19)
    s.cap, s.scores = cap, hydra.Scores(cap)
    s.q.copy_((s.q.float() * sign * cap).to(BF16))  # scores of deviation one cap
    O, L, rq, rkv = s.reference()
    sh = s.share()
    ring.forward(sh, s.q, s.kv)
    vmax = float(s.kv[0][1].float().abs().max())
    # weights are as far off as the scores: 2^-16 A of |q| |k| / sqrt(192) at most some 12 caps, 2^-19 of a cap; the sums of
    # weights and values besides
    off = 12 * 2.0 ** -16 * cap + 2.0 ** -18 * cap
    assert np.abs(sh.o_acc.cpu().numpy() - O).max() <= (1.1 * 2.0 ** -8 + 2 * off) * vmax
    assert np.abs(sh.lse_acc.cpu().numpy() - L).max() <= off + 2.0 ** -20 * np.abs(L).max()
    dq, dkv = s.grads()
    ring.backward(sh, s.q, s.kv, s.do, dq, dkv)
    torch.cuda.synchronize()
    if cap < 1:  # at the largest, one key takes a row's whole weight, and the gradients are roundings
        _check_grads((dq, dkv), (rq, rkv), cap)
    s.q.fill_(300.0 * sign)
    s.kv[0][0].fill_(300.0)
    ring.forward(sh, s.q, s.kv)
    torch.cuda.synchronize()
    want = cap * sign + np.log(np.arange(1, n + 1))
    assert np.abs(sh.lse_acc.cpu().numpy()[0] - want).max() <= 2.0 ** -20 * (cap + 8)


@pytest.mark.parametrize("case", ["tile_ends", "odd", "aligned_gqa"])
def test_plain_gradients_against_this_oracle(case):
    """The library's plain backward against the modified scores' oracle with nothing on."""
    s = Setup(case, "prefix", seed=23)
    s.prefix = None
    O, L, rq, rkv = s.reference()
    sh = s.share(scores=False)
    ring.forward(sh, s.q, s.kv)
    _check_forward(s, sh, O, L, "plain")
    dq, dkv = s.grads()
    ring.backward(sh, s.q, s.kv, s.do, dq, dkv)
    torch.cuda.synchronize()
    # D from the bf16 O, P to bf16 ahead of dS: two roundings more than the modified scores' kernels have
    for name, x, y in [("dQ", dq, rq)] + [(n, a, b) for p, r in zip(dkv, rkv) for n, a, b in zip(("dK", "dV"), p, r)]:
        x = x.double().cpu().numpy()
        assert np.linalg.norm(x - y) <= 4 * 2.0 ** -8 * np.linalg.norm(y) + 2.0 ** -18 * math.sqrt(x.size), name


def test_shares_of_scheduled_ranks():
    """Every rank of a batch that is split over heads (two to four ranks) and over a ring, with the model's slopes, a cap
    and the batch's prefixes: each rank's outputs are those of the unsplit documents' rows and heads."""
    lens, H, cap, prefix = [900, 300, 40, 17], 4, 20.0, [200, 300, 0, 5]
    mb, st, sz, _ = hydra.schedule(lens, 8, 160, pp=1)
    slopes = torch.tensor([0.25, 0.0, 0.002, -0.001], device="cuda")
    g = torch.Generator(device="cuda").manual_seed(29)
    docs = [[torch.randn((n, H, d), generator=g, device="cuda") for d in (192, 192, 128, 128)] for n in lens]
    heads_seen = set()
    for m in range(int(mb.max()) + 1):
        for r in range(8):
            share = placement.rank_share(lens, mb, st, sz, m, r, H)
            if share is None:
                continue
            hs = slice(share.head0, share.head0 + share.n_heads)
            heads_seen.add((share.head0, share.n_heads))
            probs = placement.problems(share, softcap=cap, slopes=slopes, prefix=prefix)
            for part, ps in zip(share.parts, probs):
                window = [torch.cat([docs[i][t] for i in part.seqs])[:, hs] for t in range(4)]
                rows = lambda segs: torch.cat([torch.arange(a, a + n) for a, n in segs])  # noqa: E731
                s = Setup((np.diff(part.cu).tolist(), share.n_heads, share.n_kv_heads, part.q_segs, part.kv_steps), "cap")
                s.cap, s.slopes, s.prefix, s.scores = cap, slopes[hs], [prefix[i] for i in part.seqs], ps[0].scores
                at = rows(part.q_segs)
                s.q, s.do = (window[t][at].to(BF16) for t in (0, 3))
                s.kv = [tuple(window[t][rows(step)].to(BF16) for t in (1, 2)) for step in part.kv_steps]
                O, L, rq, rkv = s.reference()
                sh = s.share()
                for p, q in zip(sh.problems, ps):
                    assert hydra.workspace_size(p) == hydra.workspace_size(q) and hydra.visible_pairs(p) == hydra.visible_pairs(q)
                sh.problems = ps
                ring.forward(sh, s.q, s.kv)
                _check_forward(s, sh, O, L, (m, r))
                dq, dkv = s.grads()
                ring.backward(sh, s.q, s.kv, s.do, dq, dkv)
                torch.cuda.synchronize()
                _check_grads((dq, dkv), (rq, rkv), (m, r))
    assert {(h, 1) for h in range(H)} <= heads_seen and (2, 2) in heads_seen


def test_timed_launches_carry_their_names():
    s = Setup("aligned_gqa", "cap")
    sh, stored = s.share(), s.share(True)
    rope = hydra.Rope()
    pos = torch.arange(s.nq, dtype=torch.int32, device="cuda")
    hydra.profile_start()
    ring.forward(sh, s.q, s.kv)
    for x in (sh, stored):
        dq, dkv = s.grads()
        ring.backward(x, s.q, s.kv, s.do, dq, dkv) if x is sh else hydra.attn_bwd_ds(
            x.problems[0], s.q, *s.kv[0], sh.o_acc, sh.lse_acc, s.do, dq, *dkv[0], x.ds_buf, x.workspace)
    hydra.rope_q(rope, s.q, pos, torch.empty_like(s.q))
    names = set(hydra.profile_stop())
    assert {"attn_fwd_scores", "bwd_pre", "bwd_recompute_scores", "bwd_dkdv_ds_scores", "bwd_dq_ds_scores", "rope_q"} <= names
    assert hydra.profile_stop() == {}
