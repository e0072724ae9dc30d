"""Linear attention and the head norm without a GPU: the oracles' pins, the plan, the checks of arguments (nothing here
reaches a kernel), and the pieces of documents that a scheduled rank holds."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import linear as L
from oracle import norm as N
from paper_2609_34318_amd import hydra, placement

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_34318_amd", "csrc")
INVALID, UNSUPPORTED, ALIGN, WORKSPACE = -1, -2, -3, -4


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not os.path.exists(hydra.LIB_PATH):
        from paper_2609_34318_amd import build_lib
        build_lib.build()
    return hydra.lib()


# ------------------------------------------------------------------ the oracles

def _inputs(seed=0, T=17, H=4, Hk=2, dk=5, dv=3, n=3):
    r = np.random.default_rng(seed).standard_normal
    return r((T, H, dk)), r((T, Hk, dk)), r((T, Hk, dv)), -np.abs(r(H)), r((T, H, dv)), r((n, H, dk, dv)), r((n, H, dk, dv))


CU = [0, 6, 6, 17]


def test_recurrence_is_the_sum_over_earlier_rows():
    q, k, v, g, _, S0, _ = _inputs()
    o, last = L.forward(CU, q, k, v, g, 0.3, S0)
    for s in range(3):
        for h in range(4):
            a, b, m = CU[s], CU[s + 1], h // 2
            i = np.arange(b - a)
            w = np.where(i[:, None] >= i, np.exp(g[h] * (i[:, None] - i)), 0.0)
            want = 0.3 * ((q[a:b, h] @ k[a:b, m].T * w) @ v[a:b, m] + np.exp(g[h] * (i + 1))[:, None] * (q[a:b, h] @ S0[s, h]))
            np.testing.assert_allclose(o[a:b, h], want, atol=1e-12)
            to_end = np.exp(g[h] * (b - a - 1 - i))[:, None]
            np.testing.assert_allclose(last[s, h], np.exp(g[h] * (b - a)) * S0[s, h] + k[a:b, m].T @ (to_end * v[a:b, m]), atol=1e-12)


def test_recurrence_gradients_against_autograd():
    q, k, v, g, do, S0, dS = _inputs(1)
    t = [torch.tensor(x, requires_grad=True) for x in (q, k, v, S0)]
    loss = 0
    lam = torch.tensor(np.exp(g))[:, None, None]
    for s in range(3):
        S = t[3][s]
        for i in range(CU[s], CU[s + 1]):
            S = lam * S + t[1][i].repeat_interleave(2, 0)[:, :, None] * t[2][i].repeat_interleave(2, 0)[:, None]
            loss = loss + 0.3 * (t[0][i][:, :, None] * S * torch.tensor(do[i])[:, None]).sum()
        loss = loss + (S * torch.tensor(dS[s])).sum()
    loss.backward()
    for x, y in zip(t, L.backward(CU, q, k, v, g, do, 0.3, S0, dS)):
        np.testing.assert_allclose(x.grad.numpy(), y, atol=1e-11)


def test_states_join_the_pieces_of_a_document():
    q, k, v, g, _, _, _ = _inputs(2)
    o, last = L.forward([0, 17], q, k, v, g)
    o1, s1 = L.forward([0, 9], q[:9], k[:9], v[:9], g)
    o2, s2 = L.forward([0, 8], q[9:], k[9:], v[9:], g, state_in=s1)
    np.testing.assert_allclose(np.concatenate([o1, o2]), o, atol=1e-12)
    np.testing.assert_allclose(s2, last, atol=1e-12)
    _, alone = L.forward([0, 8], q[9:], k[9:], v[9:], g)
    np.testing.assert_allclose(np.exp(8 * g)[:, None, None] * s1 + alone, last, atol=1e-12)


@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("activation", ["silu", "sigmoid"])
def test_norm_oracle_against_autograd(center, gated, activation):
    r = np.random.default_rng(0).standard_normal
    x, w, b, gate, dy = r((5, 3, 16)), r((3, 16)), r((3, 16)), r((5, 3, 16)) if gated else None, r((5, 3, 16))
    y, *_ = N.forward(x, w, b, gate, center, activation)
    tx, tw, tb, tg = (None if t is None else torch.tensor(t, requires_grad=True) for t in (x, w, b, gate))
    z = tx - tx.mean(-1, keepdim=True) if center else tx
    z = z / torch.sqrt((z * z).mean(-1, keepdim=True) + 1e-5) * tw + tb
    f = torch.nn.functional.silu if activation == "silu" else torch.sigmoid
    out = z * f(tg) if gated else f(z)
    np.testing.assert_allclose(out.detach().numpy(), y, atol=1e-12)
    (out * torch.tensor(dy)).sum().backward()
    dx, dg, dw, db = N.backward(x, dy, w, b, gate, center, activation)
    for t, want in ((tx, dx), (tw, dw), (tb, db), (tg, dg)):
        if t is not None:
            np.testing.assert_allclose(t.grad.numpy(), want, atol=1e-10)


# ------------------------------------------------------------------ the plan

@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_plans_cover_every_row(tmp_path):
    exe = str(tmp_path / "linear_plan")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-Wall",
           f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}", os.path.join(ROOT, "tests", "linear_plan.cpp"),
           os.path.join(CSRC, "linear_plan.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


@pytest.mark.parametrize("name", ["hydra_linear.h", "hydra_norm.h"])
def test_headers_compile_as_c_and_cpp(name, tmp_path):
    for lang, std in (("c", "c99"), ("c++", "c++11")):
        src = tmp_path / ("x." + ("c" if lang == "c" else "cpp"))
        src.write_text(f'#include "{name}"\nint main(void) {{ return 0; }}\n')
        r = subprocess.run(["gcc", "-x", lang, f"-std={std}", "-pedantic", "-Wall", "-Werror", f"-I{os.path.join(ROOT, 'include')}",
                            "-fsyntax-only", str(src)], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr


# ------------------------------------------------------------------ refusals (addresses that the host does not read)

A = 1 << 20


def _fwd(p, q=A, k=2 * A, v=3 * A, decay=4 * A, s_in=None, o=5 * A, s_out=None, ws=64 * A, n=1 << 40, planned=0):
    return hydra.lib().hydra_linear_fwd(p.ref, q, k, v, decay, s_in, o, s_out, ws, n, planned, None)


def _bwd(p, q=A, k=2 * A, v=3 * A, decay=4 * A, s_in=None, do=5 * A, ds_out=None, dq=6 * A, dk=7 * A, dv=8 * A, ds_in=None,
         ws=64 * A, n=1 << 40, planned=0):
    return hydra.lib().hydra_linear_bwd(p.ref, q, k, v, decay, s_in, do, ds_out, dq, dk, dv, ds_in, ws, n, planned, None)


def test_linear_refusals():
    p = hydra.Linear([0, 30, 50], 2, 64, 64)
    size = hydra.linear_workspace_size(p)
    assert size > 0
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(decay=None), dict(o=None), dict(o=A), dict(o=2 * A), dict(s_out=A),
               dict(s_out=5 * A), dict(o=64 * A), dict(s_in=5 * A), dict(s_in=64 * A), dict(s_in=10 * A, s_out=10 * A + 64),
               dict(decay=5 * A + 8)):
        assert _fwd(p, **kw) == INVALID, kw
    for kw in (dict(q=A + 8), dict(o=5 * A + 4), dict(decay=4 * A + 2), dict(s_in=9 * A + 4), dict(s_out=9 * A + 8), dict(ws=64 * A + 8)):
        assert _fwd(p, **kw) == ALIGN, kw
    for kw in (dict(ws=None), dict(n=size - 1), dict(planned=1), dict(planned=1, s_in=10 * A, s_out=10 * A)):
        assert _fwd(p, **kw) == WORKSPACE, kw
    for kw in (dict(q=None), dict(do=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(decay=None), dict(dq=A), dict(dk=6 * A),
               dict(dv=5 * A), dict(ds_out=9 * A, ds_in=9 * A), dict(ds_in=6 * A), dict(dk=64 * A), dict(s_in=6 * A)):
        assert _bwd(p, **kw) == INVALID, kw
    for kw in (dict(dk=7 * A + 8), dict(ds_in=9 * A + 4), dict(do=5 * A + 2)):
        assert _bwd(p, **kw) == ALIGN, kw
    for kw in (dict(ws=None), dict(n=size - 1), dict(planned=1)):
        assert _bwd(p, **kw) == WORKSPACE, kw
    for bad in (hydra.Linear([0, 4], 0), hydra.Linear([0, 4], 4, n_kv_heads=3), hydra.Linear([0, 4], 4, 100, 64),
                hydra.Linear([0, 4], 4, 64, 192), hydra.Linear([0, 4, 3], 2), hydra.Linear([1, 4], 2),
                hydra.Linear([0, 1 << 30, (1 << 30) + 1], 1), hydra.Linear(range(1 << 14), 4096, 64, 64)):
        assert hydra.linear_workspace_size(bad) == 0 and _fwd(bad) in (INVALID, UNSUPPORTED)
    for cu in ([0], [0.5, 2], [0, 1 << 31], [[0, 1]]):
        with pytest.raises(ValueError):
            hydra.Linear(cu, 2)
    # no rows and no states: nothing to do
    assert _fwd(hydra.Linear([0, 0], 2), q=None, k=None, v=None, o=None) == 0


def test_step_refusals():
    L_ = hydra.lib()

    def step(n=2, slots=3, H=2, Hk=0, dk=64, dv=64, scale=0.0, q=A, k=2 * A, v=3 * A, decay=4 * A, s=5 * A, s2=5 * A, sl=6 * A, o=7 * A):
        return L_.hydra_linear_step(n, slots, H, Hk, dk, dv, scale, q, k, v, decay, s, s2, sl, o, None)
    for kw in (dict(n=-1), dict(n=65537), dict(slots=-1), dict(H=0), dict(H=4097), dict(H=4, Hk=3), dict(H=2, Hk=4), dict(dk=0),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(sl=None, slots=1), dict(q=None), dict(k=None), dict(v=None),
               dict(decay=None), dict(s=None), dict(s2=None), dict(o=None), dict(o=A), dict(o=5 * A), dict(s2=5 * A + 64), dict(s2=A),
               dict(s2=6 * A), dict(n=65536, slots=65536, H=4096)):
        assert step(**kw) == INVALID, kw
    for kw in (dict(dk=96), dict(dv=192), dict(dv=32)):
        assert step(**kw) == UNSUPPORTED, kw
    for kw in (dict(q=A + 8), dict(s=5 * A + 4, s2=5 * A + 4), dict(sl=6 * A + 2), dict(decay=4 * A + 1)):
        assert step(**kw) == ALIGN, kw
    assert step(n=0, q=None, k=None, v=None, o=None) == 0


def test_norm_refusals():
    L_ = hydra.lib()

    def make(T=4, H=2, d=64, u=1, center=1, act=1, eps=1e-5):
        return ctypes.byref(hydra.NormC(T, H, d, u, center, act, eps))

    def fwd(p=None, x=A, w=2 * A, b=3 * A, g=4 * A, y=5 * A, **kw):
        return L_.hydra_unpack_heads_normed(p or make(**kw), x, w, b, g, y, None)

    def bwd(p=None, x=A, w=2 * A, b=3 * A, g=4 * A, dy=5 * A, dx=6 * A, dg=7 * A, dw=8 * A, db=9 * A, ws=64 * A, n=1 << 30, **kw):
        return L_.hydra_pack_heads_normed_bwd(p or make(**kw), x, w, b, g, dy, dx, dg, dw, db, ws, n, None)
    for kw in (dict(T=-1), dict(T=(1 << 31) + 1), dict(H=0), dict(H=65537), dict(d=4), dict(d=96), dict(d=1024), dict(u=0), dict(H=3, u=2),
               dict(act=2), dict(act=-1), dict(eps=0.0), dict(eps=-1.0), dict(eps=1e-39), dict(eps=float("inf")), dict(eps=float("nan"))):
        assert fwd(**kw) == INVALID and bwd(**kw) == INVALID, kw
    for kw in (dict(x=None), dict(y=None), dict(y=A), dict(y=4 * A), dict(y=2 * A)):
        assert fwd(**kw) == INVALID, kw
    for kw in (dict(x=A + 8), dict(w=2 * A + 4), dict(g=4 * A + 2)):
        assert fwd(**kw) == ALIGN, kw
    for kw in (dict(x=None), dict(dy=None), dict(dx=None), dict(dg=None), dict(g=None), dict(w=None), dict(b=None), dict(dx=A), dict(dg=6 * A),
               dict(dw=9 * A), dict(db=2 * A), dict(ws=6 * A)):
        assert bwd(**kw) == INVALID, kw
    size = hydra.norm_workspace_size(4, 2, 64)
    for kw in (dict(ws=None), dict(n=size - 1), dict(dw=None, ws=None)):
        assert bwd(**kw) == WORKSPACE, kw
    for kw in (dict(dx=6 * A + 8), dict(ws=64 * A + 4), dict(dw=8 * A + 4)):
        assert bwd(**kw) == ALIGN, kw
    assert hydra.norm_workspace_size(4, 2, 96) == 0 and hydra.norm_workspace_size(-1, 2, 64) == 0
    assert fwd(T=0, x=None, y=None) == 0 and bwd(T=0, x=None, dy=None, dx=None, dw=None, db=None) == 0
    with pytest.raises(ValueError):
        hydra.unpack_heads_normed(torch.zeros((1, 2, 1, 64), dtype=torch.bfloat16), None, activation="relu")


# ------------------------------------------------------------------ a scheduled rank's pieces

def test_scheduled_ranks_hold_every_document_once():
    lens = [700, 64, 3000, 128, 512]
    mb, st, sz, _ = hydra.schedule(lens, 8, 2048)
    rows = {d: np.zeros(n, int) for d, n in enumerate(lens)}
    for m in range(int(max(mb)) + 1):
        for r in range(8):
            share = placement.rank_share(lens, mb, st, sz, m, r, 8)
            if share is None or share.u:  # ranks of one group over heads hold the same rows
                continue
            for part in share.parts:
                p, pieces = placement.linear(share, part, 64, 64)
                assert list(np.diff(p.cu)) == [n for _, _, n in pieces] and p.n_tokens == sum(n for _, n in part.q_segs)
                assert hydra.linear_workspace_size(p) > 0
                sc = placement.scores(share, part, window=100, sinks=2)
                assert sc.window == 100 and sc.sinks == 2 and placement.scores(share, part) is None
                for d, first, n in pieces:
                    rows[part.seqs[d]][first:first + n] += 1
    assert all((x == 1).all() for x in rows.values())
