"""Modified scores and rotary positions without a GPU: the oracle's pins, the plan of prefixes, the checks of
arguments (nothing here reaches a kernel), the constants of the cap, and what a scheduled rank's share takes."""
import ctypes
import math
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import attention as A
from oracle import scores as S
from paper_2609_34318_amd import hydra, placement, ring

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_34318_amd", "csrc")


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not os.path.exists(hydra.LIB_PATH):
        from paper_2609_34318_amd import build_lib
        build_lib.build()
    return hydra.lib()


# ------------------------------------------------------------------ the oracle

def _tensors(rng, nq, nk, H, Hkv, d=24, dv=16):
    return rng.standard_normal((nq, H, d)), rng.standard_normal((nk, Hkv, d)), rng.standard_normal((nk, Hkv, dv))


CU, Q_SEGS, STEPS, PREFIX = [0, 7, 7, 20, 31], [(2, 9), (15, 16)], [[(0, 12)], [(12, 5), (25, 6)], [(17, 8)]], [3, 0, 13, 5]


@pytest.mark.parametrize("softcap,slopes,prefix", [(0, None, None), (2.0, None, None), (0, [0.5, -0.1, 0.0, 2.0], None),
                                                   (0, None, PREFIX), (1.5, [0.3, 0.1, 0.0, 1.0], PREFIX)])
def test_oracle_against_autograd(softcap, slopes, prefix):
    """Every formula of the oracle from torch's derivatives, ring steps merged and summed."""
    rng = np.random.default_rng(0)
    nq, H, Hkv = 25, 4, 2
    k_segs = [s for st in STEPS for s in st]
    q, k, v = _tensors(rng, nq, 31, H, Hkv)
    do = rng.standard_normal((nq, H, 16))
    kw = dict(scale=0.3, softcap=softcap, slopes=slopes, prefix=prefix)
    O, L = S.attn_fwd(q, k, v, CU, Q_SEGS, k_segs, **kw)
    tq, tk, tv = (torch.tensor(x, requires_grad=True) for x in (q, k, v))
    qp, kp = torch.tensor(A.row_positions(Q_SEGS)), torch.tensor(A.row_positions(k_segs))
    vis = torch.tensor(S.visible(CU, Q_SEGS, k_segs, prefix))
    s = 0.3 * torch.einsum("qhd,khd->hqk", tq, tk.repeat_interleave(2, 1))
    if softcap:
        s = softcap * torch.tanh(s / softcap)
    if slopes is not None:
        s = s - torch.tensor(slopes, dtype=torch.float64)[:, None, None] * (qp[:, None] - kp[None]).abs()
    s = s.masked_fill(~vis, -math.inf)
    o = torch.einsum("hqk,khd->qhd", torch.softmax(s, -1), tv.repeat_interleave(2, 1))
    np.testing.assert_allclose(o.detach().numpy(), O, atol=1e-12)
    np.testing.assert_allclose(torch.logsumexp(s, -1).detach().numpy(), L, atol=1e-12)
    (o * torch.tensor(do)).sum().backward()
    dQ, row, mO, mL = np.zeros(q.shape), 0, None, None
    for st in STEPS:
        n = sum(m for _, m in st)
        ks, vs = k[row:row + n], v[row:row + n]
        part = S.attn_fwd(q, ks, vs, CU, Q_SEGS, st, **kw)
        mO, mL = part if mO is None else A.lse_merge(mO, mL, *part)
        a, b, c = S.attn_bwd(q, ks, vs, O, L, do, CU, Q_SEGS, st, **kw)
        dQ += a
        np.testing.assert_allclose(tk.grad.numpy()[row:row + n], b, atol=1e-11)
        np.testing.assert_allclose(tv.grad.numpy()[row:row + n], c, atol=1e-11)
        row += n
    np.testing.assert_allclose(tq.grad.numpy(), dQ, atol=1e-11)
    np.testing.assert_allclose(mO, O, atol=1e-12)
    np.testing.assert_allclose(mL, L, atol=1e-12)


def test_oracle_without_modification_is_the_plain_oracle():
    rng = np.random.default_rng(1)
    q, k, v = _tensors(rng, 25, 17, 4, 2)
    do = rng.standard_normal((25, 4, 16))
    segs = [(12, 5), (0, 12)]
    O, L = S.attn_fwd(q, k, v, CU, Q_SEGS, segs)
    O2, L2 = A.attn_fwd(q, k, v, CU, Q_SEGS, segs)
    np.testing.assert_allclose(O, O2, atol=1e-13)
    np.testing.assert_allclose(L, L2, atol=1e-13)
    for a, b in zip(S.attn_bwd(q, k, v, O, L, do, CU, Q_SEGS, segs), A.attn_bwd(q, k, v, O, L, do, CU, Q_SEGS, segs)):
        np.testing.assert_allclose(a, b, atol=1e-12)


def test_oracle_gradient_by_differences():
    rng = np.random.default_rng(2)
    q, k, v = _tensors(rng, 25, 31, 2, 1)
    do = rng.standard_normal((25, 2, 16))
    segs = [(0, 31)]
    kw = dict(scale=0.4, softcap=1.2, slopes=[0.2, 0.05], prefix=PREFIX)
    loss = lambda q, k, v: (S.attn_fwd(q, k, v, CU, Q_SEGS, segs, **kw)[0] * do).sum()  # noqa: E731
    O, L = S.attn_fwd(q, k, v, CU, Q_SEGS, segs, **kw)
    grads = S.attn_bwd(q, k, v, O, L, do, CU, Q_SEGS, segs, **kw)
    for x, g in zip((q, k, v), grads):
        step = rng.standard_normal(x.shape)
        e = 1e-6
        args = lambda sign: [y + sign * e * step if y is x else y for y in (q, k, v)]  # noqa: E731
        diff = (loss(*args(1)) - loss(*args(-1))) / (2 * e)
        assert abs(diff - (g * step).sum()) <= 1e-7 * (np.abs(g * step).sum() + 1)


@pytest.mark.parametrize("pairing", ["interleaved", "halves", "axis_halves"])
def test_rotation_oracle(pairing):
    """A rotation keeps lengths, its inverse undoes it, and products of rotated rows depend on the
    difference of their positions alone."""
    rng = np.random.default_rng(3)
    pairs = S.rope_pairs([3, 5], pairing, "axis")
    cols = np.concatenate(pairs[:2])
    assert sorted(cols) == list(range(16))
    x, y = rng.standard_normal((2, 6, 2, 16))
    p = rng.integers(-1000, 1000, (2, 6))
    r = S.rotate(x, p, pairs)
    np.testing.assert_allclose((r ** 2).sum(-1), (x ** 2).sum(-1))
    np.testing.assert_allclose(S.rotate(r, p, pairs, inverse=True), x, atol=1e-12)
    dot = (S.rotate(x, p, pairs) * S.rotate(y, p + 5, pairs)).sum(-1)
    np.testing.assert_allclose(dot, (S.rotate(x, p - 70, pairs) * S.rotate(y, p - 65, pairs)).sum(-1), atol=1e-9)


# ------------------------------------------------------------------ plan

def _random_problem(rng):
    nd = int(rng.integers(1, 14))
    lens = [int(rng.choice([0, 1, 5, rng.integers(0, 400), rng.integers(0, 60)])) for _ in range(nd)]
    lens[0] = max(lens[0], 1)
    cu = np.concatenate([[0], np.cumsum(lens)])
    prefix = [int(rng.choice([0, n, rng.integers(0, n + 1)])) for n in lens]

    def segs():
        out = []
        for _ in range(int(rng.integers(0, 5))):
            a = int(rng.integers(0, cu[-1] + 1))
            out.append((a, int(rng.integers(0, cu[-1] - a + 1))))
        return out
    return cu, prefix, segs(), segs()


def test_plan_covers_the_visible_pairs():
    rng = np.random.default_rng(4)
    for trial in range(250):
        cu, prefix, q, k = _random_problem(rng)
        p = hydra.Problem(cu, 2, q, k, scores=hydra.Scores(prefix=prefix))
        vis = S.visible(cu, q, k, prefix)
        assert hydra.visible_pairs(p) == vis.sum()
        for which, V in ((0, vis), (1, vis.T)):
            cover = np.zeros(V.shape, int)
            for it in hydra.plan_items(p, which):
                for r in range(it[3]):
                    cover[it[0]:it[0] + it[2], it[4 + 3 * r]:it[4 + 3 * r] + it[6 + 3 * r]] += 1
            assert cover.max(initial=0) <= 1 and (cover[V] == 1).all(), (trial, which)


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_stored_ds_slots_of_prefixes(tmp_path):
    exe = str(tmp_path / "scores_plan")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-Wall",
           f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}", os.path.join(ROOT, "tests", "scores_plan.cpp"),
           os.path.join(CSRC, "plan.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


def test_nothing_on_is_the_plain_problem():
    q = [(100, 900)]
    for n_kv in (0, 1):
        a = hydra.Problem([0, 400, 1000], 4, q, q, n_kv_heads=n_kv)
        b = hydra.Problem([0, 400, 1000], 4, q, q, n_kv_heads=n_kv, scores=hydra.Scores())
        for f in (hydra.workspace_size, hydra.split_scratch_size, hydra.visible_pairs, lambda p: hydra.bwd_ds_bytes(p, 1)):
            assert f(a) == f(b)
        for which in (0, 1):
            assert np.array_equal(hydra.plan_items(a, which), hydra.plan_items(b, which))
    L = hydra.lib()
    p = hydra.Problem([0, 64], 1, [(0, 64)], [(0, 64)])
    assert L.hydra_scores_workspace_size(p.ref, None) == L.hydra_workspace_size(p.ref)


# ------------------------------------------------------------------ refusals

def _ptrs(n, step=1 << 30):
    """Disjoint aligned addresses that are never dereferenced."""
    return [(i + 1) * step for i in range(n)]


def test_scores_are_checked_on_the_host():
    L = hydra.lib()
    p = hydra.Problem([0, 64, 128], 2, [(0, 128)], [(0, 128)])
    def size(cap=0.0, slopes=None, prefix=None, scale=0.0):
        s = hydra.Scores(cap, None, prefix)
        s.c.slopes = slopes
        p.c.softmax_scale = scale
        return L.hydra_scores_workspace_size(p.ref, ctypes.byref(s.c))
    ok = size()
    assert ok > 0 and size(50.0) >= ok and size(slopes=1 << 20) >= ok and size(prefix=[64, 0]) >= ok
    for cap in (-1.0, math.nan, math.inf, 2.0 ** -11, 2.0 ** 11):
        assert size(cap) == 0, cap
    assert size(2.0 ** -10) > 0 and size(2.0 ** 10) > 0
    assert size(1.0, scale=2048.0) == 0 and size(2.0, scale=2048.0) > 0         # scale / cap above 2^10
    assert size(512.0, scale=2.0 ** -6) == 0 and size(256.0, scale=2.0 ** -6) > 0  # below 2^-14
    assert size(1.0, scale=2.0 ** -9) == 0 and size(1.0, scale=2.0 ** -8) > 0
    assert size(slopes=(1 << 20) + 2) == 0                               # not 4-byte aligned
    assert size(slopes=(1 << 20) + 4) > 0                                # 16 bytes are not asked of a slice
    assert size(prefix=[65, 0]) == 0 and size(prefix=[0, -1]) == 0
    p.c.softmax_scale = 0.0
    q, k, v, o, lse, ws, of, lf, do, dq, dk, dv, ds = _ptrs(13)
    s = hydra.Scores(50.0)
    s.c.slopes = lse + 4
    fwd = lambda sc, **kw: L.hydra_scores_fwd(p.ref, ctypes.byref(sc.c), kw.get("q", q), k, v, o, kw.get("lse", lse), None,  # noqa: E731
                                              kw.get("ws", ws), kw.get("n", 1 << 29), None, 0, 0, 1, None)
    assert fwd(s) == -1                                   # the slopes lie in an output
    s.c.slopes = 1 << 20
    assert fwd(s, q=None) == -1 and fwd(s, q=q + 8) == -3 and fwd(s, n=16) == -4 and fwd(s, ws=None) == -4
    assert fwd(s) == -4                                   # planned, and nothing was planned there
    s.c.softcap = -1.0
    assert fwd(s) == -1
    s.c.softcap = 50.0

    def bwd(o_bytes=4, ds_buf=None, planned=1, **kw):
        return L.hydra_scores_bwd(p.ref, ctypes.byref(s.c), q, k, v, kw.get("of", of), o_bytes, lf, do, kw.get("dq", dq), dk,
                                  dv, ds_buf, 1 << 20 if ds_buf else 0, ws, 1 << 29, None, 0, planned, None)
    assert bwd(o_bytes=3) == -1 and bwd(o_bytes=0) == -1
    assert bwd(ds_buf=ds) == -1                           # planned with stored dS
    assert bwd(dq=1 << 20) == -1                          # the slopes lie in a gradient
    # an fp32 O is twice as long: here its second half is dQ
    n = 128 * 2 * 128 * 2
    assert bwd(o_bytes=4, dq=of + n) == -1 and bwd(o_bytes=2, dq=of + n) == -4
    assert bwd() == -4
    r = hydra.Problem([0, 64, 128], 2, [(0, 128)], [(0, 128)], scores=hydra.Scores(50.0))
    with pytest.raises(ValueError):
        hydra.attn_bwd_noalloc(r, *[None] * 9)


def test_binding_refuses_scores():
    with pytest.raises(ValueError, match="device tensor"):
        hydra.Scores(slopes=torch.zeros(2))
    with pytest.raises(ValueError, match="prefix"):
        hydra.Problem([0, 5, 9], 1, [(0, 9)], [(0, 9)], scores=hydra.Scores(prefix=[1]))
    for prefix in ([1.5], [2 ** 32 + 5], np.array([2 ** 32 + 5]), [float("nan")]):
        with pytest.raises((ValueError, OverflowError)), np.errstate(invalid="ignore"):
            hydra.Scores(prefix=prefix)
    for cap in (1e-46, -1e-50):  # 0 in 32 bits, which would be no cap
        with pytest.raises(ValueError, match="softcap"):
            hydra.Scores(softcap=cap)
    with pytest.raises(hydra.HydraError):
        ring.make_share([0, 5], 1, [(0, 5)], [[(0, 5)]], device="cpu", scores=hydra.Scores(softcap=-3.0))


def _rope(pairs=(32,), **kw):
    r = hydra.Rope(pairs)
    for name, x in kw.items():
        setattr(r.c, name, x)
    r.keep = kw
    return r


def test_rope_arguments_are_checked_on_the_host():
    L = hydra.lib()
    src, pos, dst, kv, pe, k, v, g, h, dkv, dpe = _ptrs(11)

    def q(r=None, T=8, H=8, d=192, u=4, src=src, stride=0, pos=pos, dst=dst):
        return L.hydra_rope_q((r or _rope()).ref, T, H, d, u, src, stride, pos, dst, None)
    assert q(T=0) == 0 and q(T=0, src=None, pos=None, dst=None) == 0
    for kw in (dict(T=-1), dict(T=(1 << 30) + 1), dict(H=0), dict(H=4097), dict(u=0), dict(u=3), dict(d=56), dict(d=520),
               dict(d=196), dict(src=None), dict(pos=None), dict(dst=None), dict(stride=8 * 192 - 8),
               dict(stride=8 * 192 + 4), dict(stride=1 << 30), dict(dst=src), dict(dst=src + 16), dict(dst=pos + 16),
               dict(dst=pos, u=1)):
        assert q(**kw) == -1, kw
    for kw in (dict(src=src + 8), dict(pos=pos + 2), dict(dst=dst + 2)):
        assert q(**kw) == -3, kw
    inf = (ctypes.c_double * 32)(*[math.inf] * 32)
    for r in (_rope(n_axes=0), _rope(n_axes=5), _rope(pairing=3), _rope(pairing=-1), _rope(per_axis=2),
              _rope(base=0.5, inv_freq=None), _rope(base=math.nan, inv_freq=None), _rope(base=math.inf, inv_freq=None),
              _rope(inv_freq=ctypes.cast(inf, ctypes.POINTER(ctypes.c_double))), _rope(pairs=[30]), _rope(pairs=[132]),
              _rope(pairs=[100, 32]), _rope(pairs=[0, 32])):
        assert q(r, T=0) == -1
    assert q(_rope(pairs=[100, 28]), T=0, d=256) == 0

    def kvf(T=8, H=8, n=128, dv=128, u=4, kv=kv, s=0, pe=pe, ps=0, pos=pos, k=k, v=v):
        return L.hydra_rope_kv(_rope().ref, T, H, n, dv, u, kv, s, pe, ps, pos, k, v, None)
    assert kvf(T=0) == 0 and kvf(T=0, dv=0, v=None) == 0
    for kw in (dict(n=-8), dict(n=132), dict(dv=-8), dict(dv=4), dict(n=456), dict(n=256, dv=264), dict(kv=None),
               dict(pe=None), dict(k=None), dict(v=None), dict(s=8), dict(ps=56), dict(k=v), dict(k=kv + 16),
               dict(v=pe), dict(v=pos + 16), dict(u=5)):
        assert kvf(**kw) == -1, kw
    assert kvf(pe=pe + 8) == -3

    def qb(T=8, d=192, gb=4, g=g, pos=pos, dst=dst, stride=0, u=4):
        return L.hydra_rope_q_bwd(_rope().ref, T, 8, d, u, gb, g, pos, dst, stride, None)
    assert qb(T=0) == 0
    for kw in (dict(gb=1), dict(gb=8), dict(d=56), dict(g=None), dict(dst=g), dict(dst=pos), dict(stride=16), dict(u=16)):
        assert qb(**kw) == -1, kw
    # the fp32 gradient is 8 * 8 * 192 * 4 bytes long, the bf16 one half of it
    assert qb(dst=g + 8 * 8 * 192 * 4 - 16) == -1

    def kb(T=8, n=128, dv=128, gb=4, dk=g, dvp=h, pos=pos, dkv=dkv, s=0, dpe=dpe, ps=0, u=4):
        return L.hydra_rope_kv_bwd(_rope().ref, T, 8, n, dv, u, gb, dk, dvp, pos, dkv, s, dpe, ps, None)
    assert kb(T=0) == 0 and kb(T=0, dv=0, dvp=None) == 0
    for kw in (dict(gb=3), dict(dk=None), dict(dvp=None), dict(dkv=None), dict(dpe=None), dict(dkv=dpe), dict(dkv=g),
               dict(dpe=h), dict(dpe=pos), dict(s=8), dict(ps=8), dict(n=130), dict(n=460, dv=0)):
        assert kb(**kw) == -1, kw
    assert kb(dpe=dpe + 8) == -3
    # both in the rows of one buffer: their columns may not meet (where they do not, the GPU tests run it)
    row = 8 * 256 + 64
    for at in (8 * 256 - 8, 8 * 256 + 8, -56, 0, 3 * row + 8 * 256 - 8, row - 8):
        assert kb(dpe=dkv + 2 * at, s=row, ps=row) == -1
    assert kb(dpe=dkv + 2 * 8 * 256, s=row, ps=row + 8) == -1


def test_binding_refuses_rope_tensors():
    for kw in (dict(pairs=[]), dict(pairs=[1] * 5), dict(pairing="x"), dict(ladder="x"), dict(inv_freq=[1.0])):
        with pytest.raises(ValueError):
            hydra.Rope(**kw)


# ------------------------------------------------------------------ constants of the cap

def test_polynomial_of_the_cap():
    """s (poly[0] + poly[1] s^2 + ...) in 32 bits, as the kernels evaluate it, against out tanh(s scale / c), where out
    is c log2(e) in the forward and 1 in the backward, and the shorter one of small scores: seven roundings of half a step each on top of the fit's 6e-7, over scores up to the polynomial's range."""
    text = open(os.path.join(CSRC, "kernels.h")).read()
    numbers = lambda name: [float(x) for x in re.search(name + r" = \{?(.*?)\}?;", text).group(1).split(",")]  # noqa: E731
    f = np.float32
    for cap, scale in ((50.0, 192 ** -0.5), (30.0, 1.0), (2.0 ** 10, 2.0 ** -4), (2.0 ** -10, 1.0), (2.0 ** 6, 2.0 ** -8),
                       (2.0 ** 10, 2.0 ** 20)):
        into = scale / cap
        for out, name, n, end in ((cap * math.log2(math.e), "TANH_POLY", 5, "TANH_NEAR"), (1.0, "TANH_POLY", 5, "TANH_NEAR"),
                                  (cap * math.log2(math.e), "TANH_LOW", 3, "TANH_SMALL"), (1.0, "TANH_LOW", 3, "TANH_SMALL")):
            poly, (near,) = numbers(name + rf"\[{n}\]"), numbers(end)
            c = [f(poly[k] * into * out * into ** (2 * k)) for k in range(n)]
            s = np.linspace(0, near / into, 20001)[1:].astype(f)
            w = s * s
            r = f(c[n - 1]) * w + f(c[n - 2])
            for k in reversed(range(n - 2)):
                r = r * w + f(c[k])
            got = (r * s).astype(np.float64)
            want = out * np.tanh(s.astype(np.float64) * into)
            assert np.abs(got / want - 1).max() <= 6e-7 + 7 * 2.0 ** -24


# ------------------------------------------------------------------ a scheduled rank's share

def test_scores_and_positions_of_a_rank_share():
    lens = [96, 40, 300, 17, 260]
    mb, st, sz, _ = hydra.schedule(lens, 4, 256, pp=1)
    prefix = [5, 40, 0, 3, 260]
    seen = set()
    for m in range(int(mb.max()) + 1):
        for r in range(4):
            share = placement.rank_share(lens, mb, st, sz, m, r, 8)
            if share is None:
                continue
            for part, probs in zip(share.parts, placement.problems(share, softcap=30.0, prefix=prefix)):
                assert placement.scores(share, part) is None
                assert all(p.scores.softcap == 30.0 and list(p.scores.prefix) == [prefix[i] for i in part.seqs]
                           for p in probs)
                pos = placement.doc_positions(part, part.q_segs)
                want = [a + i - max(c for c in part.cu if c <= a + i) for a, n in part.q_segs for i in range(n)]
                assert pos.dtype == np.int32 and list(pos) == want
                seen |= set(part.seqs)
    assert seen == set(range(5))
    assert len(placement.doc_positions(part, [])) == 0
