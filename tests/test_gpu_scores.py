"""GPU parity of attention with modified scores (cap, distance bias, prefix mask) against the fp64 oracle.

Tolerances, from the roundings that the kernels make (a rounding to bf16 is off by at most 2^-8 of the value, to
fp16 by 2^-11, to fp32 by 2^-24):
  O    its weights are rounded to bf16: 2^-8 of the largest |v|, and 10% for everything in 32 bits; the bf16 copy
       once more
  LSE  scores are 32-bit sums of 192 exact products, each off by at most 2^-24 of the sum of their magnitudes
       so far; bounded by 1e-4 for unit inputs, times q's scale; biases are 32-bit values: 2^-21 of the largest |LSE|
  dQ, dK, dV  relative L2: dS (or P) is rounded to bf16 once, D and P carry O's and fp16's errors: 2 * 2^-8
"""
import math

import numpy as np
import pytest
import torch

from oracle import attention as A
from oracle import scores as S
from paper_2609_34318_amd import hydra, ring

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
TOL_GRAD = 2 * 2.0 ** -8

CASES = {
    # documents, query heads, K/V heads, query segments, K/V segments of every step
    "odd": ([5, 0, 65, 33], 3, 3, [(0, 103)], [[(0, 103)]]),
    "one_token": ([1], 2, 2, [(0, 1)], [[(0, 1)]]),
    "ring_rows_that_see_nothing": ([40, 300, 60], 4, 2, [(0, 400)], [[(150, 120)], [(0, 150), (390, 10)], [(270, 120)]]),
    "aligned_gqa": ([100, 412], 8, 2, [(0, 512)], [[(0, 512)]]),
    "aligned_zigzag": ([640], 2, 2, [(0, 160), (480, 160)], [[(0, 160), (480, 160)], [(160, 160), (320, 160)]]),
    "many_documents": ([1 + (7 * i) % 9 for i in range(90)], 2, 1, [(3, 400)], [[(0, 200)], [(200, 250)]]),
    "last_rows": ([3000], 2, 1, [(2995, 5)], [[(0, 3000)]]),
    "tile_ends": ([257, 129], 1, 1, [(0, 386)], [[(0, 257)], [(257, 129)]]),
}
MODS = {
    # cap, slopes by head, prefix (a share of every document, or lengths), q's scale
    "cap": (50.0, None, None, 1.0),
    "cap_reached": (1.5, None, None, 4.0),
    "bias": (0.0, "ladder", None, 1.0),
    "bias_negative": (0.0, "negative", None, 1.0),
    "prefix": (0.0, None, 0.5, 1.0),
    "prefix_all": (0.0, None, 1.0, 1.0),
    "all": (8.0, "ladder", 0.4, 3.0),
    "all_no_prefix": (20.0, "ladder", None, 1.0),
}


def _slopes(kind, H):
    if kind is None:
        return None
    s = [2.0 ** (-8.0 * (h + 1) / H) for h in range(H)]
    return torch.tensor([-x / 64 for x in s] if kind == "negative" else s, dtype=F32, device="cuda")


def _prefix(share, docs):
    return None if share is None else [int(round(share * n)) if i % 3 else (n if share == 1.0 else 0) for i, n in enumerate(docs)]


class Setup:
    def __init__(self, case, mod, seed=0, graph_ready=False, heads=None):
        docs, H, Hkv, q_segs, steps = CASES[case] if isinstance(case, str) else case
        cap, slopes, prefix, qs = MODS[mod]
        self.cu = [0] + list(np.cumsum(docs))
        self.H, self.Hkv, self.q_segs, self.steps, self.q_scale = H, Hkv, q_segs, steps, qs
        self.slopes, self.prefix, self.cap = _slopes(slopes, H), _prefix(prefix, docs), cap
        self.scores = hydra.Scores(cap, self.slopes, self.prefix)
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        nq = sum(n for _, n in q_segs)
        self.q = (r(nq, H, 192) * qs).to(BF16)
        self.kv = [(r(sum(n for _, n in s), Hkv, 192).to(BF16), (r(sum(n for _, n in s), Hkv, 128) / 11).to(BF16)) for s in steps]
        self.do = r(nq, H, 128).to(BF16)
        self.nq = nq
        self.graph_ready = graph_ready

    def share(self, ds=False, scratch=True, scores=True):
        sh = ring.make_share(self.cu, self.H, self.q_segs, self.steps, n_kv_heads=self.Hkv, graph_ready=self.graph_ready,
                             scores=self.scores if scores else None, ds_kv_heads=1 if ds else 0)
        if not scratch:
            sh.scratch = None
        for t in (sh.o_acc, sh.lse_acc, sh.o_bf16):
            t.fill_(math.nan)
        return sh

    def grads(self):
        z = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
        return z(self.nq, self.H, 192), [(z(k.shape[0], self.Hkv, 192), z(k.shape[0], self.Hkv, 128)) for k, _ in self.kv]

    def kw(self):
        return dict(softcap=self.cap, slopes=None if self.slopes is None else self.slopes.cpu().numpy(), prefix=self.prefix)

    def reference(self):
        f = lambda t: t.float().cpu().numpy()  # noqa: E731
        union = [s for st in self.steps for s in st]
        q, do = f(self.q), f(self.do)
        kv = [(f(k), f(v)) for k, v in self.kv]
        O, L = S.attn_fwd(q, np.concatenate([k for k, _ in kv]), np.concatenate([v for _, v in kv]), self.cu, self.q_segs,
                          union, **self.kw())
        dq, dkv = np.zeros(q.shape), []
        for st, (k, v) in zip(self.steps, kv):
            a, b, c = S.attn_bwd(q, k, v, O, L, do, self.cu, self.q_segs, st, **self.kw())
            dq += a
            dkv.append((b, c))
        return O, L, dq, dkv


def _n(t):
    return t.float().cpu().numpy().astype(np.float64)


def _check_forward(s, sh, O, L, what):
    vmax = max(float(v.float().abs().max()) for _, v in s.kv)
    o, o16, lse = _n(sh.o_acc), _n(sh.o_bf16), _n(sh.lse_acc)
    assert np.isfinite(o).all() and np.isfinite(o16).all(), what
    assert np.abs(o - O).max() <= 1.1 * 2.0 ** -8 * vmax, what
    assert np.abs(o16 - O).max() <= 2.1 * 2.0 ** -8 * vmax, what
    empty = np.isneginf(L)
    assert np.array_equal(np.isneginf(lse), empty) and not o[empty.T].any(), what
    if not empty.all():
        assert np.abs(lse[~empty] - L[~empty]).max() <= 1e-4 * s.q_scale + 2.0 ** -21 * np.abs(L[~empty]).max(), what


def _check_grads(got, ref, what):
    dq, dkv = got
    rq, rkv = ref
    pairs = [("dQ", dq, rq)]
    for i, ((a, b), (c, d)) in enumerate(zip(dkv, rkv)):
        pairs += [(f"dK {i}", a, c), (f"dV {i}", b, d)]
    for name, x, y in pairs:
        x = _n(x)
        assert np.isfinite(x).all(), (what, name)
        # a row that sees one key has no gradient but the rounding of dP - D
        err, norm = np.linalg.norm(x - y), np.linalg.norm(y)
        assert err <= TOL_GRAD * norm + 2.0 ** -18 * math.sqrt(x.size), (what, name, err / max(norm, 1e-30))


@pytest.mark.parametrize("mod", MODS)
@pytest.mark.parametrize("case", CASES)
def test_parity(case, mod):
    """Forward with its merges, the recompute backward, with and without scratch, and the stored-dS one."""
    s = Setup(case, mod)
    O, L, rq, rkv = s.reference()
    for scratch, ds in ((True, False), (False, False), (True, True)):
        sh = s.share(ds, scratch)
        if ds and sh.ds_buf is None:
            continue
        ring.forward(sh, s.q, s.kv)
        _check_forward(s, sh, O, L, (scratch, ds))
        dq, dkv = s.grads()
        ring.backward(sh, s.q, s.kv, s.do, dq, dkv)
        torch.cuda.synchronize()
        _check_grads((dq, dkv), (rq, rkv), (scratch, ds))
        # again: the same bits, and the gradients added
        first = [t.clone() for t in (sh.o_acc, sh.lse_acc, sh.o_bf16, dq, *[x for p in dkv for x in p])]
        ring.forward(sh, s.q, s.kv)
        dq, dkv = s.grads()
        ring.backward(sh, s.q, s.kv, s.do, dq, dkv)
        again = [sh.o_acc, sh.lse_acc, sh.o_bf16, dq, *[x for p in dkv for x in p]]
        assert all(torch.equal(a, b) for a, b in zip(first, again))
    assert not case.startswith("aligned") or s.share(True).ds_buf is not None


def test_bf16_output_for_the_backward():
    """D from the bf16 O, as a program that kept only that has it; the fp32 O is nearer to the oracle."""
    s = Setup("aligned_gqa", "all", seed=3)
    O, L, rq, rkv = s.reference()
    sh = s.share()
    ring.forward(sh, s.q, s.kv)
    p, (k, v), err = sh.problems[0], s.kv[0], {}
    for o in (sh.o_bf16, sh.o_acc):
        dq, dkv = s.grads()
        hydra.attn_bwd(p, s.q, k, v, o, sh.lse_acc, s.do, dq, *dkv[0], sh.workspace, scratch=sh.scratch)
        torch.cuda.synchronize()
        _check_grads((dq, dkv), (rq, rkv), o.dtype)
        err[o.dtype] = np.linalg.norm(_n(dq) - rq)
    assert err[F32] < err[BF16]


@pytest.mark.parametrize("case", ["odd", "aligned_gqa", "ring_rows_that_see_nothing"])
def test_nothing_on_is_the_plain_call(case):
    s = Setup(case, "cap")
    s.scores = hydra.Scores()
    out = []
    for scores in (True, False):
        sh = s.share(scores=scores)
        ring.forward(sh, s.q, s.kv)
        dq, dkv = s.grads()
        for p, (k, v), (dk, dv) in zip(sh.problems, s.kv, dkv):
            hydra.attn_bwd(p, s.q, k, v, sh.o_bf16, sh.lse_acc, s.do, dq, dk, dv, sh.workspace, scratch=sh.scratch)
        out.append([sh.o_acc, sh.lse_acc, sh.o_bf16, dq, *[x for q in dkv for x in q]])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*out))


@pytest.mark.parametrize("case,mod", [("ring_rows_that_see_nothing", "all"), ("aligned_zigzag", "cap"),
                                      ("many_documents", "prefix")])
def test_recorded_step_replays(case, mod):
    """A recorded step (forward, merges, backward) against the eager one on new inputs and new slopes before every
    replay, with eager calls on the same problems between them."""
    s = Setup(case, mod, graph_ready=True)
    sh, eager = s.share(), s.share()
    ring.plan(sh)
    dq, dkv = s.grads()
    tensors = [dq] + [x for p in dkv for x in p]

    def step():
        ring.forward(sh, s.q, s.kv, planned=True)
        for t in tensors:
            t.zero_()
        ring.backward(sh, s.q, s.kv, s.do, dq, dkv, planned=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        g = torch.Generator(device="cuda").manual_seed(100 + i)
        s.q.copy_(torch.randn(s.q.shape, generator=g, device="cuda"))
        if s.slopes is not None:
            s.slopes.copy_(torch.rand(s.slopes.shape, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = [sh.o_acc, sh.lse_acc, sh.o_bf16] + [t.clone() for t in tensors]
        ring.forward(eager, s.q, s.kv)
        eq, ekv = s.grads()
        ring.backward(eager, s.q, s.kv, s.do, eq, ekv)
        torch.cuda.synchronize()
        want = [eager.o_acc, eager.lse_acc, eager.o_bf16, eq] + [x for p in ekv for x in p]
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i


def test_plans_of_other_scores_are_refused():
    """The prefixes are part of a plan, the cap and the slopes are not."""
    seg = [(0, 96)]
    make = lambda **kw: hydra.Problem([0, 40, 96], 2, seg, seg, scores=hydra.Scores(**kw) if kw else None)  # noqa: E731
    base = make(prefix=[10, 0])
    ws = torch.empty(hydra.workspace_size(base), dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(0)
    q, k = (torch.randn((96, 2, 192), generator=g, device="cuda").to(BF16) for _ in range(2))
    v = torch.randn((96, 2, 128), generator=g, device="cuda").to(BF16)
    o, lse = torch.empty((96, 2, 128), device="cuda"), torch.empty((2, 96), device="cuda")
    run = lambda p: hydra.attn_fwd(p, q, k, v, o, lse, ws, planned=True)  # noqa: E731
    hydra.attn_plan(base, ws)
    run(base)
    run(make(prefix=[10, 0], softcap=5.0))
    run(make(prefix=[10, 0], slopes=torch.ones(2, device="cuda")))
    for p in (make(), make(prefix=[11, 0]), make(softcap=5.0)):
        with pytest.raises(hydra.HydraError) as e:
            run(p)
        assert e.value.status == -4
    hydra.attn_plan(make(), ws)
    for p in (base, make(softcap=5.0)):
        with pytest.raises(hydra.HydraError) as e:
            run(p)
        assert e.value.status == -4
    run(make())
    torch.cuda.synchronize()


def test_no_rows_need_no_tensors():
    for scores in (None, hydra.Scores(30.0)):
        p = hydra.Problem([0, 8], 2, [], [(0, 8)], scores=scores)
        ws = torch.empty(max(1, hydra.workspace_size(p)), dtype=torch.uint8, device="cuda")
        k = torch.zeros((8, 2, 192), dtype=BF16, device="cuda")
        dk = torch.ones((8, 2, 192), device="cuda")
        dv = torch.ones((8, 2, 128), device="cuda")
        hydra.attn_bwd(p, None, k, k[..., :128].contiguous(), None, None, None, None, dk, dv, ws)
        torch.cuda.synchronize()
        assert float(dk.min()) == 1 and float(dv.max()) == 1


def test_tensors_elsewhere_are_refused():
    p = hydra.Problem([0, 8], 2, [(0, 8)], [(0, 8)], scores=hydra.Scores(30.0))
    ws = torch.empty(hydra.workspace_size(p), dtype=torch.uint8, device="cuda")
    q = torch.zeros((8, 2, 192), dtype=BF16, device="cuda")
    v = torch.zeros((8, 2, 128), dtype=BF16, device="cuda")
    o, lse = torch.empty((8, 2, 128), device="cuda"), torch.empty((2, 8), device="cuda")
    with pytest.raises(ValueError):
        hydra.attn_fwd(p, q.cpu(), q, v, o, lse, ws)
    with pytest.raises(ValueError):
        hydra.attn_fwd(p, q, q[:, :1].expand(8, 2, 192), v, o, lse, ws)
    with pytest.raises(ValueError, match="slopes"):
        hydra.Problem([0, 8], 2, [(0, 8)], [(0, 8)], scores=hydra.Scores(slopes=torch.zeros(3, device="cuda")))
    with pytest.raises(ValueError, match="dtype"):
        hydra.Scores(slopes=torch.zeros(2, device="cuda", dtype=BF16))
    plain = hydra.Problem([0, 8], 2, [(0, 8)], [(0, 8)])
    with pytest.raises(ValueError, match="o_final"):  # without modified scores the final O is bf16
        hydra.attn_bwd(plain, q, q, v, o, lse, v, *(torch.zeros((8, 2, d), device="cuda") for d in (192, 192, 128)), ws)


@pytest.mark.parametrize("mod", ["all", "prefix"])
def test_views_of_fused_buffers(mod):
    """q, k and v as slices of wider rows, and a view of the model's slopes that is not 16-byte aligned."""
    s = Setup("odd", mod)
    dense = s.share()
    ring.forward(dense, s.q, s.kv)
    dq, dkv = s.grads()
    ring.backward(dense, s.q, s.kv, s.do, dq, dkv)
    fused = torch.randn((s.nq, s.H * 512 + 8), device="cuda").to(BF16)
    k, v = s.kv[0]
    views = []
    for t, at in ((s.q, 0), (k, s.H * 192), (v, s.H * 384)):
        d = t.shape[-1]
        w = fused[:, at:at + s.H * d].unflatten(1, (s.H, d))
        w.copy_(t)
        views.append(w)
    if s.slopes is not None:
        model = torch.cat([torch.full((1,), math.nan, device="cuda"), s.slopes])
        s.scores = hydra.Scores(s.cap, model[1:], s.prefix)
        assert s.scores.c.slopes % 16
    sh = s.share()
    ring.forward(sh, views[0], [(views[1], views[2])])
    eq, ekv = s.grads()
    ring.backward(sh, views[0], [(views[1], views[2])], s.do, eq, ekv)
    torch.cuda.synchronize()
    for a, b in ((dense.o_acc, sh.o_acc), (dense.lse_acc, sh.lse_acc), (dq, eq), (dkv[0][0], ekv[0][0]), (dkv[0][1], ekv[0][1])):
        assert torch.equal(a, b)


@pytest.mark.parametrize("mod", ["all", "cap_reached"])
def test_rows_past_32_bit_offsets(mod):
    """Token rows 2^21 elements apart: the last ones lie beyond 2^31 elements, the same bits as dense."""
    n, pitch = 1100, 1 << 21
    s = Setup(([700, 400], 1, 1, [(0, n)], [[(0, n)]]), mod)
    dense = s.share()
    ring.forward(dense, s.q, s.kv)
    dq, dkv = s.grads()
    ring.backward(dense, s.q, s.kv, s.do, dq, dkv)
    wide = torch.empty((n, pitch), dtype=BF16, device="cuda")
    q, k = wide[:, :192].unsqueeze(1), wide[:, 1024:1024 + 192].unsqueeze(1)
    q.copy_(s.q)
    k.copy_(s.kv[0][0])
    sh = s.share()
    kv = [(k, s.kv[0][1])]
    ring.forward(sh, q, kv)
    eq, ekv = s.grads()
    ring.backward(sh, q, kv, s.do, eq, ekv)
    torch.cuda.synchronize()
    for a, b in ((dense.o_acc, sh.o_acc), (dq, eq), (dkv[0][0], ekv[0][0]), (dkv[0][1], ekv[0][1])):
        assert torch.equal(a, b)


def test_far_positions_and_distances():
    """A document that starts beyond 2^30, and one of 2^25 tokens whose last rows see its prefix and themselves:
    distances beyond what 32-bit floats count by one."""
    far = (1 << 30) + 5
    for docs, q_segs, steps, prefix in (
            ([far, 300], [(far, 300)], [[(far, 150)], [(far + 150, 150)]], [0, 70]),
            ([1 << 25], [((1 << 25) - 64, 64)], [[(0, 96), ((1 << 25) - 64, 64)]], [1000])):
        s = Setup((docs, 2, 1, q_segs, steps), "all")
        s.prefix = prefix
        s.slopes.copy_(torch.tensor([0.25, 1e-7]))
        s.scores = hydra.Scores(s.cap, s.slopes, prefix)
        O, L, rq, rkv = s.reference()
        sh = s.share()
        ring.forward(sh, s.q, s.kv)
        _check_forward(s, sh, O, L, docs)
        dq, dkv = s.grads()
        ring.backward(sh, s.q, s.kv, s.do, dq, dkv)
        torch.cuda.synchronize()
        _check_grads((dq, dkv), (rq, rkv), docs)


def test_extreme_scores():
    """Scores far beyond the cap (the weights of capped ties are equal), slopes that leave each row itself
    alone, and caps at both ends of their range."""
    n = 200
    s = Setup(([n], 1, 1, [(0, n)], [[(0, n)]]), "cap_reached")
    s.q.fill_(300.0)
    s.kv[0][0].fill_(300.0)
    for cap in (2.0 ** -6, 5.0, 2.0 ** 10):
        s.cap, s.scores = cap, hydra.Scores(cap)
        sh = s.share()
        ring.forward(sh, s.q, s.kv)
        torch.cuda.synchronize()
        want = cap * math.tanh(300 * 300 * 192 ** 0.5 / cap) + np.log(np.arange(1, n + 1))
        assert np.abs(_n(sh.lse_acc)[0] - want).max() <= 2.0 ** -20 * (cap + 8)
        dq, dkv = s.grads()
        ring.backward(sh, s.q, s.kv, s.do, dq, dkv)
        torch.cuda.synchronize()
        # a score at its cap does not move: 1 - tanh^2 is what three 32-bit roundings of tanh^2 leave, 2^-22, of
        # gradients of at most 192^-1/2 * |dP - D| * 300, which a key sums over its n rows
        left = 2.0 ** -22 * 192 ** -0.5 * 300 * 2 * float((s.do.float().abs().sum(-1).max() * s.kv[0][1].float().abs().max()))
        assert float(dq.abs().max()) <= left and float(dkv[0][0].abs().max()) <= n * left
        assert torch.isfinite(dkv[0][1]).all()
    s = Setup(([n], 1, 1, [(0, n)], [[(0, n)]]), "bias")
    s.slopes.fill_(1e30)
    sh = s.share()
    ring.forward(sh, s.q, s.kv)
    dq, dkv = s.grads()
    ring.backward(sh, s.q, s.kv, s.do, dq, dkv)
    torch.cuda.synchronize()
    assert torch.equal(sh.o_acc, s.kv[0][1].float())
    assert torch.equal(dkv[0][1], s.do.float())
    assert float(dq.abs().max()) <= 2.0 ** -18 and float(dkv[0][0].abs().max()) <= 2.0 ** -18


def test_forwards_of_one_plan_overlap():
    """Two streams on one planned workspace with slopes of their own."""
    s = Setup("aligned_gqa", "all", graph_ready=True)
    other = torch.rand(s.H, device="cuda")
    sh = s.share()
    ring.plan(sh)
    b = hydra.Problem(s.cu, s.H, s.q_segs, s.steps[0], n_kv_heads=s.Hkv, scores=hydra.Scores(s.cap, other, s.prefix))
    k, v = s.kv[0]
    out = []
    for _ in range(2):
        row = []
        for p, stream in ((sh.problems[0], torch.cuda.Stream()), (b, torch.cuda.Stream())):
            o, lse = torch.empty((s.nq, s.H, 128), device="cuda"), torch.empty((s.H, s.nq), device="cuda")
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                for _ in range(4):
                    hydra.attn_fwd(p, s.q, k, v, o, lse, sh.step_workspaces[0], planned=True)
            row.append((o, lse, stream))
        torch.cuda.synchronize()
        out.append(row)
    for (o, lse, _), (o2, lse2, _) in zip(*out):
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
    assert not torch.equal(out[0][0][0], out[0][1][0])


@pytest.mark.parametrize("mod", ["cap", "all"])
def test_gradients_by_differences(mod):
    """The backward against differences of the oracle's forward along random directions."""
    s = Setup(([60, 40], 2, 1, [(0, 100)], [[(0, 100)]]), mod, seed=5)
    sh = s.share()
    ring.forward(sh, s.q, s.kv)
    dq, dkv = s.grads()
    ring.backward(sh, s.q, s.kv, s.do, dq, dkv)
    torch.cuda.synchronize()
    f = lambda t: t.float().cpu().numpy().astype(np.float64)  # noqa: E731
    x = [f(s.q), f(s.kv[0][0]), f(s.kv[0][1])]
    loss = lambda y: (S.attn_fwd(*y, s.cu, s.q_segs, s.steps[0], **s.kw())[0] * f(s.do)).sum()  # noqa: E731
    rng = np.random.default_rng(0)
    for i, g in enumerate((dq, *dkv[0])):
        d = rng.standard_normal(x[i].shape)
        e = 1e-5
        diff = (loss([y + e * d if j == i else y for j, y in enumerate(x)]) -
                loss([y - e * d if j == i else y for j, y in enumerate(x)])) / (2 * e)
        g = _n(g)
        # along a direction the error's part is its norm over that of a random direction
        assert abs(diff - (g * d).sum()) <= 6 * TOL_GRAD * np.linalg.norm(g), i


def test_shared_oracle_of_the_plain_call():
    """The library's plain call against this oracle with nothing on: the two are held to one definition."""
    s = Setup("tile_ends", "prefix")
    s.prefix = None
    O, L, rq, rkv = s.reference()
    sh = s.share(scores=False)
    ring.forward(sh, s.q, s.kv)
    _check_forward(s, sh, O, L, "plain")
    qp = A.row_positions(s.q_segs)
    assert len(qp) == s.nq


@pytest.mark.parametrize("mod,ds", [("all", False), ("cap", True), ("prefix", True), ("bias", False)])
def test_many_tiles(mod, ds):
    """Eight heads on four (whole heads per XCD), items of tens of tiles, prefixes over several of them."""
    s = Setup(([1472, 2048], 8, 4, [(0, 3520)], [[(0, 3520)]]), mod, seed=9)
    O, L, rq, rkv = s.reference()
    sh = s.share(ds)
    assert (sh.ds_buf is not None) == ds
    ring.forward(sh, s.q, s.kv)
    _check_forward(s, sh, O, L, mod)
    dq, dkv = s.grads()
    ring.backward(sh, s.q, s.kv, s.do, dq, dkv)
    torch.cuda.synchronize()
    _check_grads((dq, dkv), (rq, rkv), mod)
