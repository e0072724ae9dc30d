"""The head norm with an activation or a gate against the fp64 oracle, element by element.

Tolerances, derived: an output rounded to bf16 is off by half a step, 2^-8 of itself.  Before that a value has sums of at
most 512 terms in a tree (3 + 6 additions in a row, each off by 2^-24 of what is summed), a reciprocal square root, an
exp2 and a reciprocal of 2^-22 each, and a dozen products: under 2^-18 of the sum A of its terms' magnitudes.  Sums over
T tokens round once per token more: T 2^-24 of their terms' magnitudes.
"""
import numpy as np
import pytest
import torch

from oracle import norm as oracle
from paper_2609_34318_amd import hydra

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def draw(seed, T, H, d, cp_u, weight, bias, gate, scale=1.0, shift=0.0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    x = (r(cp_u, T, H // cp_u, d) * scale + shift).to(BF16)
    return dict(x=x, d_y=r(T, H, d).to(BF16), weight=1 + 0.3 * r(H, d) if weight else None, bias=0.3 * r(H, d) if bias else None,
                gate=(2 * r(T, H, d)).to(BF16) if gate else None)


def run(x, center=True, activation="silu", eps=1e-5, backward=True):
    c = {n: None if t is None else t.cuda() for n, t in x.items()}
    u, T, Hg, d = x["x"].shape
    new = lambda t, dt=None: None if t is None else torch.full(t.shape, 7.0, dtype=dt or t.dtype, device="cuda")  # noqa: E731
    how = dict(weight=c["weight"], bias=c["bias"], gate=c["gate"], center=center, activation=activation, eps=eps)
    out = {"y": new(x["d_y"])}
    hydra.unpack_heads_normed(c["x"], out["y"], **how)
    if backward:
        out.update(d_x=new(x["x"]), d_gate=new(x["gate"]), d_weight=new(x["weight"]), d_bias=new(x["bias"]))
        ws = torch.empty(hydra.norm_workspace_size(T, u * Hg, d), dtype=torch.uint8, device="cuda")
        hydra.pack_heads_normed_bwd(c["x"], c["d_y"], out["d_x"], d_gate=out["d_gate"], d_weight=out["d_weight"],
                                    d_bias=out["d_bias"], workspace=ws, **how)
    return out


def check(x, got, center, activation, eps=1e-5):
    f = lambda t: None if t is None else t.double().numpy()  # noqa: E731
    xs, w, b, g, dy = oracle.unpack(x["x"].double()), f(x["weight"]), f(x["bias"]), f(x["gate"]), f(x["d_y"])
    how = dict(weight=w, bias=b, gate=g, center=center, activation=activation, eps=eps)
    y, xn, r, z = oracle.forward(xs, **how)
    d_x, d_gate, d_w, d_b = oracle.backward(xs, dy, **how)
    # magnitudes of the terms of x', z and what follows from them
    mean = lambda t: t.mean(-1, keepdims=True)  # noqa: E731
    ax = (np.abs(xs) + (mean(np.abs(xs)) if center else 0)) * r
    aw, ab = (1.0 if w is None else np.abs(w)), (0.0 if b is None else np.abs(b))
    az = ax * aw + ab
    a, da = oracle.act(z if g is None else g, activation)
    if g is None:  # z's error goes through the activation, whose slope is at most 1.1
        ay, adz = az * 1.1 + np.abs(a), np.abs(dy) * (np.abs(da) + az)
    else:
        ay, adz = az * np.abs(a), np.abs(dy * a)
    au = adz * aw
    along = mean(au * ax)
    adx = r * (au + (mean(au) if center else 0) + ax * along)
    T = xs.shape[0]
    want = {"y": (y, ay), "d_x": (d_x, adx), "d_gate": (d_gate, None if g is None else np.abs(dy) * az * (np.abs(da) + 0.1))}
    for n, (ref, size) in want.items():
        if got.get(n) is None:
            continue
        t = got[n].double().cpu().numpy()
        t = oracle.unpack(t) if n == "d_x" else t
        tol = np.abs(ref) * 2.0 ** -8 + size * 2.0 ** -18 + 1e-30
        assert np.isfinite(t).all() and (np.abs(t - ref) <= tol).all(), (n, (np.abs(t - ref) / tol).max())
    for n, ref, size in (("d_weight", d_w, (adz * ax).sum(0)), ("d_bias", d_b, adz.sum(0))):
        if got.get(n) is not None:
            t, tol = got[n].double().cpu().numpy(), size * (2.0 ** -18 + T * 2.0 ** -24) + 1e-30
            assert (np.abs(t - ref) <= tol).all(), (n, (np.abs(t - ref) / tol).max())


SIZES = [(1, 1, 8, 1), (1, 16, 128, 1), (5, 3, 32, 3), (37, 2, 512, 2), (300, 8, 64, 4), (33, 40, 128, 8), (1027, 1, 256, 1), (9, 6, 16, 2)]


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("center", [True, False], ids=["center", "rms"])
@pytest.mark.parametrize("gate", [True, False], ids=["gate", "plain"])
@pytest.mark.parametrize("activation", ["silu", "sigmoid"])
def test_parity(size, center, gate, activation):
    T, H, d, u = size
    for weight, bias in ((True, True), (False, False), (True, False)):
        x = draw(T + d, T, H, d, u, weight, bias, gate, scale=3.0, shift=0.5)
        check(x, run(x, center, activation), center, activation)


def test_a_constant_head_and_a_far_mean():
    """Heads of one value: only eps stands under the root; and a mean 100 times the deviation."""
    x = draw(3, 20, 2, 64, 1, True, True, True, scale=0.0, shift=3.0)
    check(x, run(x), True, "silu")
    x = draw(4, 20, 2, 64, 1, True, True, True, scale=0.5, shift=50.0)
    check(x, run(x), True, "silu")
    x = draw(5, 20, 2, 64, 1, False, False, True, scale=0.0)
    got = run(x, center=False)
    assert not got["y"].any() and torch.isfinite(got["d_x"].float()).all()


@pytest.mark.parametrize("center", [True, False], ids=["center", "rms"])
def test_values_at_the_ends_of_their_range(center):
    """Up to 2^58, where the sum of 512 squares still fits 32 bits, and so small that eps alone stands under the root."""
    x = draw(7, 6, 2, 512, 1, True, True, True, scale=2.0 ** 55)
    assert 2.0 ** 56 < x["x"].abs().max() <= 2.0 ** 58
    check(x, run(x, center), center, "silu")
    x = draw(8, 6, 2, 512, 1, True, True, True, scale=2.0 ** -70)
    check(x, run(x, center), center, "silu")


def test_a_token_that_is_not_finite_stays_by_itself():
    x = draw(9, 9, 4, 32, 2, True, True, True)
    want = run(x)
    x["x"][0, 4, 1, 5], x["x"][1, 7, 0, 0] = float("nan"), float("inf")
    got = run(x)
    for n in ("y", "d_gate"):
        a, b = got[n].float(), want[n].float()
        other = torch.ones(9, 4, dtype=torch.bool)
        other[4, 1] = other[7, 2] = False  # head 0 of the second group is head 2
        assert torch.equal(a[other], b[other]) and not torch.isfinite(a[~other]).any(1).all(), n


def test_far_gates():
    x = draw(6, 8, 2, 64, 1, False, False, True)
    x["gate"] = torch.where(torch.rand(x["gate"].shape, generator=torch.Generator().manual_seed(0)) < 0.5, 3e38, -3e38).to(BF16)
    got = run(x, activation="sigmoid")
    y, _, _, z = oracle.forward(oracle.unpack(x["x"].double()), gate=x["gate"].double().numpy(), activation="sigmoid")
    assert np.abs(got["y"].double().cpu().numpy() - y).max() <= 2.0 ** -8 * np.abs(y).max()
    assert not got["d_gate"].any()


@pytest.mark.parametrize("gate", [True, False], ids=["gate", "plain"])
def test_where_a_value_that_is_not_finite_goes(gate):
    """x: its token and head (every channel) and d_weight, d_bias only where the activation is of the norm itself; d_y: its
    own channel's d_gate, its token and head of d_x, and both sums of its channel."""
    x = draw(11, 9, 4, 32, 2, True, True, gate)
    want = run(x)
    bad = {n: None if t is None else t.clone() for n, t in x.items()}
    bad["x"][0, 4, 1, 5], bad["x"][1, 7, 0, 0] = float("nan"), float("inf")
    got = run(bad)
    heads = torch.zeros(9, 4, dtype=torch.bool)
    heads[4, 1] = heads[7, 2] = True  # head 0 of the second group is head 2

    def flat(t, n):
        t = t.float().cpu()
        return torch.cat(list(t), 1) if n == "d_x" else t
    for n in ("y", "d_gate", "d_x"):
        if got[n] is not None:
            a, b = flat(got[n], n), flat(want[n], n)
            assert torch.equal(a[~heads], b[~heads]) and not torch.isfinite(a[heads]).any(), n
    of_head = heads.any(0)
    for n in ("d_weight", "d_bias"):
        a, b = got[n].cpu(), want[n].cpu()
        assert torch.equal(a[~of_head], b[~of_head]), n
        if n == "d_bias" and gate:  # the sum of d_y act(gate): x has no part in it
            assert torch.equal(a, b)
        else:
            assert not torch.isfinite(a[of_head]).any(), n
    bad = {n: None if t is None else t.clone() for n, t in x.items()}
    bad["d_y"][3, 2, 7] = float("nan")
    got = run(bad)
    assert torch.equal(got["y"], want["y"])
    heads[:] = False
    heads[3, 2] = True
    a, b = flat(got["d_x"], "d_x"), flat(want["d_x"], "d_x")
    assert torch.equal(a[~heads], b[~heads]) and not torch.isfinite(a[heads]).any()
    for n in ("d_weight", "d_bias"):
        assert torch.isfinite(got[n]).sum() == 4 * 32 - 1 and not torch.isfinite(got[n][2, 7]), n
    if gate:
        assert torch.isfinite(got["d_gate"]).sum() == 9 * 4 * 32 - 1 and not torch.isfinite(got["d_gate"][3, 2, 7])
