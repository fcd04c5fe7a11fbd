"""Norm of a head, then rotation by position (oracle, test only; fp64 NumPy).

x [R, H, d]: y = w * x / sqrt(mean(x^2) + eps) (w None: y = x); with h = len(inv_freq) and the angle
a_i = position * inv_freq_i, the pair (y_i, y_{i+h}) is turned by a_i; elements from 2h on stay.
"""
from __future__ import annotations

import numpy as np


def _angles(positions, inv_freq):
    a = np.asarray(positions, np.float64)[:, None, None] * np.asarray(inv_freq, np.float64)
    return np.cos(a), np.sin(a)


def _turn(y, cos, sin):
    h = cos.shape[-1]
    out = y.copy()
    out[..., :h] = y[..., :h] * cos - y[..., h:2 * h] * sin
    out[..., h:2 * h] = y[..., h:2 * h] * cos + y[..., :h] * sin
    return out


def norm_rope(x, weight, positions, inv_freq, eps):
    x = np.asarray(x, np.float64)
    y = x
    if weight is not None:
        y = np.asarray(weight, np.float64) * x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps)
    return _turn(y, *_angles(positions, inv_freq))


def norm_rope_grad(x, weight, positions, inv_freq, eps, dout):
    """(dx, dw or None) of sum(dout * norm_rope(x))."""
    x, dout = np.asarray(x, np.float64), np.asarray(dout, np.float64)
    cos, sin = _angles(positions, inv_freq)
    dy = _turn(dout, cos, -sin)
    if weight is None:
        return dy, None
    w = np.asarray(weight, np.float64)
    r = 1.0 / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps)
    dw = (dy * x * r).sum(axis=(0, 1))
    return r * (w * dy - x * r * r * (w * dy * x).mean(axis=-1, keepdims=True)), dw
