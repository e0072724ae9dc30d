"""fp64 oracle of the linear attention with a decay for each head: the recurrence, one token at a time.

    S_t = e^g S_{t-1} + k_t v_t^T,   o_t = scale q_t S_t

and its gradients by the reversed recurrence G_t = scale q_t^T dO_t + e^g G_{t+1}.
"""
from __future__ import annotations

import numpy as np


def _grouped(x, heads):
    return np.repeat(x, heads // x.shape[1], axis=1)


def forward(cu, q, k, v, decay, scale=0.0, state_in=None):
    """q [T, H, d_k], k, v [T, Hkv, .] -> o [T, H, d_v], states [n, H, d_k, d_v]."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    T, H, dk = q.shape
    k, v = _grouped(k, H), _grouped(v, H)
    scale = scale or 1 / np.sqrt(dk)
    lam = np.exp(np.asarray(decay, np.float64))[:, None, None]
    o = np.zeros((T, H, v.shape[2]))
    last = np.zeros((len(cu) - 1, H, dk, v.shape[2]))
    for s in range(len(cu) - 1):
        S = np.zeros(last.shape[1:]) if state_in is None else np.asarray(state_in[s], np.float64).copy()
        for t in range(cu[s], cu[s + 1]):
            S = lam * S + k[t][:, :, None] * v[t][:, None, :]
            o[t] = scale * (q[t][:, :, None] * S).sum(1)
        last[s] = S
    return o, last


def backward(cu, q, k, v, decay, d_o, scale=0.0, state_in=None, d_state_out=None):
    """dq, dk, dv (summed over the query heads of a K/V head) and the gradients of the first states."""
    q, k, v, d_o = (np.asarray(t, np.float64) for t in (q, k, v, d_o))
    T, H, dk = q.shape
    Hk = k.shape[1]
    k, v = _grouped(k, H), _grouped(v, H)
    dv = v.shape[2]
    scale = scale or 1 / np.sqrt(dk)
    lam = np.exp(np.asarray(decay, np.float64))[:, None, None]
    dq, dK, dV = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    first = np.zeros((len(cu) - 1, H, dk, dv))
    for s in range(len(cu) - 1):
        S = np.zeros((H, dk, dv)) if state_in is None else np.asarray(state_in[s], np.float64).copy()
        for t in range(cu[s], cu[s + 1]):
            S = lam * S + k[t][:, :, None] * v[t][:, None, :]
            dq[t] = scale * (S * d_o[t][:, None, :]).sum(2)
        G = np.zeros((H, dk, dv)) if d_state_out is None else np.asarray(d_state_out[s], np.float64).copy()
        for t in range(cu[s + 1] - 1, cu[s] - 1, -1):
            G = G + scale * q[t][:, :, None] * d_o[t][:, None, :]
            dK[t] = (G * v[t][:, None, :]).sum(2)
            dV[t] = (G * k[t][:, :, None]).sum(1)
            G = lam * G
        first[s] = G
    return dq, dK.reshape(T, Hk, H // Hk, dk).sum(2), dV.reshape(T, Hk, H // Hk, dv).sum(2), first
