"""fp64 oracle of the head norm with an activation or a gate: the definition, and its derivatives written out."""
from __future__ import annotations

import numpy as np


def act(t, kind):
    """The activation and its derivative."""
    e = np.exp(-np.abs(t))
    s = np.where(t >= 0, 1 / (1 + e), e / (1 + e))
    ds = e / (1 + e) ** 2
    return (s, ds) if kind == "sigmoid" else (t * s, s + t * ds)


def unpack(x):
    """[cp_u, T, H / cp_u, d] -> [T, H, d]"""
    return np.concatenate(list(np.asarray(x, np.float64)), axis=1)


def forward(x, weight=None, bias=None, gate=None, center=True, activation="silu", eps=1e-5):
    """x [T, H, d] -> y, and what the backward needs: x', r, z."""
    x = np.asarray(x, np.float64)
    if center:
        x = x - x.mean(-1, keepdims=True)
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    xn = x * r
    z = xn * (1.0 if weight is None else np.asarray(weight, np.float64)) + (0.0 if bias is None else np.asarray(bias, np.float64))
    a, _ = act(z if gate is None else np.asarray(gate, np.float64), activation)
    return (a if gate is None else z * a), xn, r, z


def backward(x, d_y, weight=None, bias=None, gate=None, center=True, activation="silu", eps=1e-5):
    """d_x, d_gate, d_weight, d_bias."""
    _, xn, r, z = forward(x, weight, bias, gate, center, activation, eps)
    d_y = np.asarray(d_y, np.float64)
    a, da = act(z if gate is None else np.asarray(gate, np.float64), activation)
    dz = d_y * (da if gate is None else a)
    u = dz * (1.0 if weight is None else np.asarray(weight, np.float64))
    d_x = u - xn * (u * xn).mean(-1, keepdims=True)
    if center:
        d_x = d_x - u.mean(-1, keepdims=True)
    return r * d_x, (None if gate is None else d_y * z * da), (dz * xn).sum(0), dz.sum(0)
