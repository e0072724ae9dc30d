"""One token at a time of linear attention, against the fp64 recurrence.

Tolerances, derived: a state is off by two 32-bit roundings and exp's (2^-22 of the old state, 2^-24 of the product); an
output is a 32-bit sum of d_k terms (d_k 2^-24 of their magnitudes, and the state's error) rounded to bf16 (2^-8).
"""
import numpy as np
import pytest
import torch

from paper_2609_34318_amd import hydra

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def draw(seed, n, slots, H, Hk, dk, dv):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    return dict(q=r(n, H, dk).to(BF16), k=r(n, Hk, dk).to(BF16), v=r(n, Hk, dv).to(BF16), decay=-(2.0 ** -(torch.arange(H) + 1.0)),
                state=4 * r(slots, H, dk, dv))


def expect(x, slots, scale=0.0):
    """Rows one after another."""
    q, k, v, S = (x[t].double().numpy() for t in ("q", "k", "v", "state"))
    H, dk = q.shape[1:]
    k, v = (np.repeat(t, H // t.shape[1], axis=1) for t in (k, v))
    S, size = S.copy(), np.abs(S)
    lam = np.exp(x["decay"].double().numpy())[:, None, None]
    o, so = np.full(q.shape[:2] + v.shape[2:], np.nan), np.zeros(q.shape[:2] + v.shape[2:])
    for i, s in enumerate(slots):
        if not 0 <= s < len(S):
            continue
        S[s] = lam * S[s] + k[i][:, :, None] * v[i][:, None]
        size[s] = lam * size[s] + np.abs(k[i][:, :, None] * v[i][:, None])
        f = scale or 1 / np.sqrt(dk)
        o[i], so[i] = f * (q[i][:, :, None] * S[s]).sum(1), f * (np.abs(q[i])[:, :, None] * size[s]).sum(1)
    return o, so, S, size


def check(x, slots, o, state, before, dk):
    want, so, S, size = expect(x, slots)
    o, state = o.double().cpu().numpy(), state.double().cpu().numpy()
    rows = ~np.isnan(want)
    assert (o[~rows] == 7.0).all(), "a padding row was written"
    tol = np.abs(want) * 2.0 ** -8 + so * (dk * 2.0 ** -24 + 2.0 ** -20)
    assert (np.abs(o - want)[rows] <= tol[rows]).all()
    assert (np.abs(state - S) <= size * 2.0 ** -20).all()
    untouched = [s for s in range(len(S)) if s not in set(slots)]
    assert np.array_equal(state[untouched], before.double().cpu().numpy()[untouched])


@pytest.mark.parametrize("dims", [(64, 64), (128, 64), (192, 64), (64, 128), (128, 128), (192, 128)], ids=lambda d: f"{d[0]}x{d[1]}")
@pytest.mark.parametrize("H,Hk", [(1, 1), (6, 3), (4, 1)])
@pytest.mark.parametrize("how", ["identity", "pool", "pool_out", "repeated"])
def test_parity(dims, H, Hk, how):
    dk, dv = dims
    n = 9
    x = draw(dk + H, n, 14, H, Hk, dk, dv)
    slots = {"identity": list(range(n)), "pool": [13, 2, -1, 7, 0, 14, 5, -2 ** 31, 6], "pool_out": [13, 2, -1, 7, 0, 2 ** 31 - 1, 5, 1, 6],
             "repeated": [3, 8, 3, 3, -1, 8, 0, 13, 3]}[how]
    c = {t: y.cuda() for t, y in x.items()}
    o = torch.full((n, H, dv), 7.0, dtype=BF16, device="cuda")
    before = c["state"].clone()
    out = torch.full_like(before, 5.0) if how == "pool_out" else None
    hydra.linear_step(c["q"], c["k"], c["v"], c["decay"], c["state"], o, state_out=out,
                      slots=None if how == "identity" else torch.tensor(slots, dtype=torch.int32, device="cuda"))
    if out is None:
        check(x, slots, o, c["state"], before, dk)
        return
    assert torch.equal(c["state"], before)
    used = [s for s in slots if 0 <= s < 14]
    assert (out[[s for s in range(14) if s not in used]] == 5.0).all()
    before[used] = out[used]
    check(x, slots, o, before, c["state"], dk)


@pytest.mark.parametrize("n", [1024, 1025, 2600])
def test_many_rows(n):
    """Slots of one, of several and of no rows, near each other and far apart."""
    x = draw(n, n, 700, 1, 1, 64, 64)
    slots = torch.randint(-50, 750, (n,), generator=torch.Generator().manual_seed(n)).tolist()
    slots[0] = slots[-1] = slots[n // 2] = 699
    c = {t: y.cuda() for t, y in x.items()}
    o = torch.full((n, 1, 64), 7.0, dtype=BF16, device="cuda")
    before = c["state"].clone()
    hydra.linear_step(c["q"], c["k"], c["v"], c["decay"], c["state"], o, slots=torch.tensor(slots, dtype=torch.int32, device="cuda"))
    check(x, slots, o, c["state"], before, 64)


def test_steps_continue_a_prompt():
    """The state that a prompt ends with, stepped on, against the whole sequence at once."""
    g = torch.Generator(device="cuda").manual_seed(5)
    T, H, dk, dv, cut = 150, 2, 128, 128, 140
    q, k, v = (torch.randn((T, H, d), generator=g, device="cuda").to(BF16) for d in (dk, dk, dv))
    decay = torch.tensor([-0.02, -0.5], device="cuda")
    whole, part = hydra.Linear([0, T], H, dk, dv), hydra.Linear([0, cut], H, dk, dv)
    o, state = torch.empty((T, H, dv), dtype=BF16, device="cuda"), torch.empty((2, 1, H, dk, dv), device="cuda")
    for p, s in ((whole, state[0]), (part, state[1])):
        ws = torch.empty(hydra.linear_workspace_size(p), dtype=torch.uint8, device="cuda")
        hydra.linear_fwd(p, q, k, v, decay, o, ws, state_out=s)
    steps = torch.empty((T - cut, H, dv), dtype=BF16, device="cuda")
    hydra.linear_fwd(whole, q, k, v, decay, o, torch.empty(hydra.linear_workspace_size(whole), dtype=torch.uint8, device="cuda"))
    # ten rows of one slot: consecutive tokens of its sequence
    hydra.linear_step(q[cut:], k[cut:], v[cut:], decay, state[1], steps, slots=torch.zeros(T - cut, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    # two roundings to bf16 and the 32-bit sums of both
    assert (steps.float() - o[cut:].float()).abs().max() <= 2.0 ** -7 * o.float().abs().max()
    assert (state[1] - state[0]).abs().max() <= 1e-4 * state[0].abs().max()
