"""The sliding window with sinks without a GPU: the oracle's pins, the plan, the checks of arguments."""
import math
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import attention as A
from oracle import scores as S
from paper_2609_34318_amd import hydra

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_34318_amd", "csrc")


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not os.path.exists(hydra.LIB_PATH):
        from paper_2609_34318_amd import build_lib
        build_lib.build()
    return hydra.lib()


@pytest.mark.parametrize("window,sinks", [(1, 0), (3, 2), (5, 0), (100, 4), (2, 100)])
def test_oracle_against_autograd(window, sinks):
    rng = np.random.default_rng(window)
    cu, segs = [0, 7, 7, 20, 31], [(0, 31)]
    q, k, v, do = (rng.standard_normal((31, h, d)) for h, d in ((4, 24), (2, 24), (2, 16), (4, 16)))
    kw = dict(scale=0.3, window=window, sinks=sinks)
    O, L = S.attn_fwd(q, k, v, cu, segs, segs, **kw)
    tq, tk, tv = (torch.tensor(x, requires_grad=True) for x in (q, k, v))
    sees = torch.zeros((31, 31), dtype=torch.bool)
    for a, b in zip(cu[:-1], cu[1:]):
        for i in range(a, b):
            for j in range(a, i + 1):
                sees[i, j] = j > i - window or j - a < sinks
    s = 0.3 * torch.einsum("qhd,khd->hqk", tq, tk.repeat_interleave(2, 1)).masked_fill(~sees, -math.inf)
    o = torch.einsum("hqk,khd->qhd", torch.softmax(s, -1), tv.repeat_interleave(2, 1))
    np.testing.assert_allclose(o.detach().numpy(), O, atol=1e-12)
    (o * torch.tensor(do)).sum().backward()
    for t, g in zip((tq, tk, tv), S.attn_bwd(q, k, v, O, L, do, cu, segs, segs, **kw)):
        np.testing.assert_allclose(t.grad.numpy(), g, atol=1e-11)


def test_oracle_of_a_wide_window_is_the_plain_one():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((3, 31, 2, 24))
    for a, b in zip(S.attn_fwd(q, k, v, [0, 11, 31], [(0, 31)], [(0, 31)], window=20), A.attn_fwd(q, k, v, [0, 11, 31], [(0, 31)], [(0, 31)])):
        np.testing.assert_allclose(a, b, atol=1e-13)


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_plans_cover_what_rows_see(tmp_path):
    exe = str(tmp_path / "window_plan")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-Wall",
           f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}", os.path.join(ROOT, "tests", "window_plan.cpp"),
           os.path.join(CSRC, "plan.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


def _problem(**kw):
    return hydra.Problem([0, 4096], 2, [(0, 4096)], [(0, 4096)], scores=hydra.Scores(**kw) if kw else None)


def test_work_grows_with_the_window():
    wide, narrow = (hydra.visible_pairs(_problem(window=w)) for w in (1024, 256))
    assert narrow == 256 * 4096 - 256 * 255 // 2
    assert 3.5 < wide / narrow < 4
    keys = lambda p: hydra.plan_items(p, 0)[:, 6].sum()  # noqa: E731
    assert keys(_problem(window=256)) < keys(_problem()) / 4
    assert hydra.bwd_ds_bytes(_problem(window=256), 1) < hydra.bwd_ds_bytes(_problem(), 1) / 4


def test_refusals():
    for kw in (dict(window=-1), dict(sinks=-1), dict(window=1 << 31), dict(window=2.5), dict(window=4, sinks=1 << 31)):
        with pytest.raises(ValueError):
            hydra.Scores(**kw)
    for kw in (dict(sinks=3), dict(window=4, prefix=[2]), dict(softcap=5.0, sinks=1)):
        assert hydra.workspace_size(_problem(**kw)) == 0
        with pytest.raises(hydra.HydraError) as e:
            hydra.visible_pairs(_problem(**kw))
        assert e.value.status == -1
    seg = [(0, 64)]
    with pytest.raises(ValueError):
        hydra.attn_bwd_noalloc(hydra.Problem([0, 64], 1, seg, seg, scores=hydra.Scores(window=8)), *[None] * 9)


def test_the_window_is_part_of_the_plan():
    for a, b in ((dict(window=300), dict(window=301)), (dict(window=300), dict(window=300, sinks=4)), (dict(window=300), dict(softcap=5.0))):
        assert not all(np.array_equal(hydra.plan_items(_problem(**a), w), hydra.plan_items(_problem(**b), w)) for w in (0, 1))
    a, b = _problem(window=300, sinks=4), _problem(window=300, sinks=4, softcap=30.0)
    assert hydra.workspace_size(a) == hydra.workspace_size(b)
    assert all(np.array_equal(hydra.plan_items(a, w), hydra.plan_items(b, w)) for w in (0, 1))


def test_sinks_alone_are_no_plain_problem():
    """Sinks without a window are refused by every call, and by the one that has no modified scores too."""
    assert hydra.Scores(sinks=3).any and not hydra.Scores().any
    with pytest.raises(ValueError, match="modified scores"):
        hydra.attn_bwd_noalloc(_problem(sinks=3), *[None] * 9)
