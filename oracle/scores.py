"""fp64 CPU oracle for attention with modified scores and for rotary positions.

TEST INFRASTRUCTURE ONLY, like the rest of this package: plain arrays in, the definitions recomputed, no code
shared with the HIP path.

Scores: for query i and key j of one document at global positions p_i and p_j,

    s_ij = tau <q_i, k_j>,  s_ij = c tanh(s_ij / c) with a cap,  s_ij = s_ij - slope_h |p_i - p_j| with slopes,

visible where p_j <= p_i or p_j lies in the document's prefix, or with a window of w keys and n sinks where p_j <= p_i
and (p_i - p_j < w or p_j is one of the document's first n).  LSE, O and D as in attention.py; backward

    dS_ij = P_ij (<dO_i, v_j> - D_i) (1 - tanh^2),  dQ = tau dS K,  dK = tau dS^T Q,  dV = P^T dO.

Rotation: pair j of columns (a, b) by the angle p f_j, p its axis' position: a' = a cos - b sin, b' = b cos + a sin.
"""
from __future__ import annotations

import math

import numpy as np

from .attention import doc_of, row_positions


def visible(cu_seqlens, q_segs, kv_segs, prefix=None, window=0, sinks=0) -> np.ndarray:
    """[Nq, Nk] truth values."""
    cu = np.asarray(cu_seqlens, dtype=np.int64)
    qp, kp = row_positions(q_segs), row_positions(kv_segs)
    if len(qp) == 0 or len(kp) == 0:
        return np.zeros((len(qp), len(kp)), bool)
    qd, kd = doc_of(cu, qp), doc_of(cu, kp)
    if window:
        near = (qp[:, None] - kp[None] < window) | (kp[None] < (cu[:-1] + sinks)[qd][:, None])
        return (qd[:, None] == kd[None]) & (kp[None] <= qp[:, None]) & near
    end = cu[:-1] + (0 if prefix is None else np.asarray(prefix, dtype=np.int64))
    return (qd[:, None] == kd[None]) & ((kp[None] <= qp[:, None]) | (kp[None] < end[qd][:, None]))


def _scores(q, k, scale, softcap, slope, qp, kp, vis):
    s = scale * (q @ k.T)
    t = np.zeros_like(s)
    if softcap:
        t = np.tanh(s / softcap)
        s = softcap * t
    if slope is not None:
        s = s - float(slope) * np.abs(qp[:, None] - kp[None]).astype(np.float64)
    return np.where(vis, s, -np.inf), 1.0 - t * t


def attn_fwd(q, k, v, cu_seqlens, q_segs, kv_segs, scale=None, softcap=0.0, slopes=None, prefix=None, window=0,
             sinks=0):
    """O [Nq, H, dv] and LSE [H, Nq] of q [Nq, H, dqk], k [Nk, Hkv, dqk], v [Nk, Hkv, dv]."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    H, grp = q.shape[1], q.shape[1] // k.shape[1]
    tau = 1.0 / math.sqrt(q.shape[2]) if scale is None else float(scale)
    vis = visible(cu_seqlens, q_segs, kv_segs, prefix, window, sinks)
    qp, kp = row_positions(q_segs), row_positions(kv_segs)
    O, L = np.zeros((q.shape[0], H, v.shape[2])), np.full((H, q.shape[0]), -np.inf)
    seen = vis.any(axis=1)
    if not seen.any():
        return O, L
    for h in range(H):
        s, _ = _scores(q[seen, h], k[:, h // grp], tau, softcap, None if slopes is None else slopes[h], qp[seen], kp,
                       vis[seen])
        m = s.max(axis=1, keepdims=True)
        e = np.exp(s - m)
        total = e.sum(axis=1, keepdims=True)
        O[seen, h] = (e / total) @ v[:, h // grp]
        L[h, seen] = (m + np.log(total))[:, 0]
    return O, L


def attn_bwd(q, k, v, o, lse, do, cu_seqlens, q_segs, kv_segs, scale=None, softcap=0.0, slopes=None, prefix=None, window=0,
             sinks=0):
    """dQ, dK, dV of one ring step from the final O and LSE of the rows."""
    q, k, v, o, lse, do = (np.asarray(x, dtype=np.float64) for x in (q, k, v, o, lse, do))
    H, grp = q.shape[1], q.shape[1] // k.shape[1]
    tau = 1.0 / math.sqrt(q.shape[2]) if scale is None else float(scale)
    vis = visible(cu_seqlens, q_segs, kv_segs, prefix, window, sinks)
    qp, kp = row_positions(q_segs), row_positions(kv_segs)
    dQ, dK, dV = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for h in range(H):
        g = h // grp
        s, f = _scores(q[:, h], k[:, g], tau, softcap, None if slopes is None else slopes[h], qp, kp, vis)
        p = np.where(vis, np.exp(np.where(vis, s - np.where(np.isfinite(lse[h]), lse[h], 0.0)[:, None], -np.inf)), 0.0)
        D = (do[:, h] * o[:, h]).sum(axis=1, keepdims=True)
        ds = p * (do[:, h] @ v[:, g].T - D) * f
        dQ[:, h] = tau * (ds @ k[:, g])
        dK[:, g] += tau * (ds.T @ q[:, h])
        dV[:, g] += p.T @ do[:, h]
    return dQ, dK, dV


# ------------------------------------------------------------------ rotary positions

def rope_pairs(pairs, pairing, ladder="whole", base=10000.0, inv_freq=None):
    """(columns a, columns b, axis, frequency) of every pair."""
    n, j0, out = sum(pairs), 0, []
    for axis, m in enumerate(pairs):
        for i in range(m):
            j = j0 + i
            a, b = {"interleaved": (2 * j, 2 * j + 1), "halves": (j, j + n), "axis_halves": (2 * j0 + i, 2 * j0 + i + m)}[
                pairing]
            f = inv_freq[j] if inv_freq is not None else base ** -(i / m if ladder == "axis" else j / n)
            out.append((a, b, axis, f))
        j0 += m
    a, b, axis, f = zip(*out)
    return np.array(a), np.array(b), np.array(axis), np.array(f, dtype=np.float64)


def rotate(x, positions, pairs, inverse=False):
    """x [T, ..., r] with its columns rotated; positions [n_axes, T]; pairs: rope_pairs()."""
    a, b, axis, f = pairs
    x = np.asarray(x, dtype=np.float64)
    angle = np.asarray(positions, dtype=np.float64)[axis].T * f
    if inverse:
        angle = -angle
    c, s = np.cos(angle), np.sin(angle)
    while c.ndim < x.ndim:
        c, s = c[:, None], s[:, None]
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y
