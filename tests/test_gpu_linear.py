"""Linear attention against the fp64 recurrence, element by element.

Tolerances, derived: with A the same recurrence over the operands' absolute values (every term of a sum counted with
its magnitude),
  - an output rounded to bf16 is off by half a step, 2^-8 of itself;
  - the forward's scores and states enter their products as sums of two bf16 values (off by 2^-16 at most), what is added to
    a state likewise, and weights are exp2 of a product rounded to 32 bits, whose error |x| 2^-24 counts e^-x of its term
    (under 2^-24): together under 2^-14 A;
  - the backward's scores and states enter as one bf16 value each, a term having one or the other: 2^-8 A more;
  - 32-bit sums round once per addend of at most three parts: 3 rows 2^-24 A, and states, which are not rounded, have
    this and the weights' error alone (2^-22 A a chunk of 32 rows).
"""
import numpy as np
import pytest
import torch

from oracle import linear as oracle
from paper_2609_34318_amd import hydra

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def draw(seed, T, H, Hk, dk, dv, n_seqs, states=True, decay=None):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    x = dict(q=r(T, H, dk).to(BF16), k=r(T, Hk, dk).to(BF16), v=r(T, Hk, dv).to(BF16), d_o=r(T, H, dv).to(BF16))
    x["decay"] = -(2.0 ** -(torch.arange(H) % 8 + 1.0)) if decay is None else torch.tensor(decay, dtype=F32)
    x["state_in"] = 3 * r(n_seqs, H, dk, dv) if states else None
    x["d_state_out"] = 0.2 * r(n_seqs, H, dk, dv) if states else None
    return x


def cuda(x):
    return {n: None if t is None else t.cuda() for n, t in x.items()}


def np64(t):
    return None if t is None else t.to(torch.float64).cpu().numpy()


def run(p, x, backward=True, workspace=None, planned=False, state_out=True):
    T = p.n_tokens
    ws = torch.empty(hydra.linear_workspace_size(p), dtype=torch.uint8, device="cuda") if workspace is None else workspace
    shape = (p.n_seqs, p.n_heads, p.d_k, p.d_v)
    out = {"o": torch.full((x["q"].shape[0], p.n_heads, p.d_v), 7.0, dtype=BF16, device="cuda"),
           "state": torch.full(shape, 7.0, device="cuda") if state_out else None}
    hydra.linear_fwd(p, x["q"], x["k"], x["v"], x["decay"], out["o"], ws, x["state_in"], out["state"], planned=planned)
    if backward:
        for n, t in (("dq", "q"), ("dk", "k"), ("dv", "v")):
            out[n] = torch.full(x[t].shape, 7.0, dtype=BF16, device="cuda")
        out["d_state"] = torch.full(shape, 7.0, device="cuda") if state_out else None
        hydra.linear_bwd(p, x["q"], x["k"], x["v"], x["decay"], x["d_o"], out["dq"], out["dk"], out["dv"], ws,
                         x["state_in"], x["d_state_out"], out["d_state"], planned=planned)
    assert T <= x["q"].shape[0]
    return out


def reference(cu, x, absolute=False):
    f = (lambda t: None if t is None else np.abs(np64(t))) if absolute else np64
    decay = np64(x["decay"])
    ins = [f(x[n])[:cu[-1]] for n in ("q", "k", "v")]
    o, last = oracle.forward(cu, *ins, decay, state_in=f(x["state_in"]))
    dq, dk, dv, first = oracle.backward(cu, *ins, decay, f(x["d_o"])[:cu[-1]], state_in=f(x["state_in"]),
                                        d_state_out=f(x["d_state_out"]))
    return {"o": o, "state": last, "dq": dq, "dk": dk, "dv": dv, "d_state": first}


def check(cu, x, got):
    want, size = reference(cu, x), reference(cu, x, absolute=True)
    rows = max([b - a for a, b in zip(cu[:-1], cu[1:])] + [1])
    for n, t in got.items():
        if t is None:
            continue
        t = np64(t)
        if n in ("state", "d_state"):
            tol = size[n] * (3 * rows * 2.0 ** -24 + (rows // 32 + 2) * 2.0 ** -22) + 1e-30
        else:
            assert (t[cu[-1]:] == 7.0).all(), f"{n}: rows behind the last sequence were written"
            t = t[:cu[-1]]
            tol = np.abs(want[n]) * 2.0 ** -8 + size[n] * (2.0 ** -14 + (0 if n == "o" else 2.0 ** -8) + 3 * rows * 2.0 ** -24) + 1e-30
        over = np.abs(t - want[n]) / tol
        assert np.isfinite(t).all() and over.max(initial=0.0) <= 1, f"{n}: {over.max()} of the tolerance at {np.unravel_index(over.argmax(), over.shape)}"


CASES = [  # rows of each sequence, H, Hkv, d_k, d_v
    ([1], 1, 1, 64, 64), ([0, 33, 0, 1, 31, 32], 2, 2, 64, 64), ([100], 3, 1, 128, 128), ([65, 2], 2, 2, 192, 128),
    ([37, 90], 4, 2, 64, 128), ([129], 2, 1, 128, 64), ([70], 2, 2, 192, 64), ([600, 5, 257], 2, 2, 128, 128),
    ([1100], 2, 1, 64, 64), ([520, 256], 1, 1, 192, 128), ([513], 2, 2, 64, 128), ([300], 2, 2, 128, 64), ([700], 1, 1, 192, 64),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[0])) + f"_h{c[1]}on{c[2]}_{c[3]}x{c[4]}")
@pytest.mark.parametrize("states", [True, False], ids=["states", "zero"])
def test_matches_the_recurrence(case, states):
    lengths, H, Hk, dk, dv = case
    cu = np.concatenate([[0], np.cumsum(lengths)])
    x = draw(sum(lengths) + dk, cu[-1] + 3, H, Hk, dk, dv, len(lengths), states)
    p = hydra.Linear(cu, H, dk, dv, n_kv_heads=Hk)
    check(cu, x, run(p, cuda(x)))
