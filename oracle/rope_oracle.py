"""Norm and rotation of query and key heads, from the definition, in fp64 numpy; positions of zigzag chunk pairs."""
from __future__ import annotations

import numpy as np

from .ring_attention_oracle import zigzag_positions  # noqa: F401  (the positions of a rank's tokens)


def pairs(rot: int, interleaved: bool):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def rotation_matrix(position: int, inv_freq, head_dim: int, interleaved: bool) -> np.ndarray:
    """[head_dim, head_dim]: the whole map, written out."""
    m = np.eye(head_dim)
    rot = 2 * len(inv_freq)
    for a, b, f in zip(*pairs(rot, interleaved), np.asarray(inv_freq, np.float64)):
        c, s = np.cos(float(position) * f), np.sin(float(position) * f)
        m[a, a], m[a, b], m[b, a], m[b, b] = c, -s, s, c
    return m


def _turn(x, positions, inv_freq, interleaved, sign):
    """x [..., token, d], positions broadcast against [..., token]."""
    y = np.array(x, np.float64)
    if len(inv_freq) == 0:
        return y
    angle = np.asarray(positions, np.float64)[..., None] * np.asarray(inv_freq, np.float64)
    c, s = np.cos(angle), sign * np.sin(angle)
    a, b = pairs(2 * len(inv_freq), interleaved)
    u, v = np.array(y[..., a]), np.array(y[..., b])
    y[..., a], y[..., b] = u * c - v * s, u * s + v * c
    return y


def rope_forward(x, weight, eps, positions, inv_freq, interleaved=False, norm=True):
    x = np.asarray(x, np.float64)
    if norm:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (1.0 if weight is None else np.asarray(weight, np.float64))
    return _turn(x, positions, inv_freq, interleaved, 1.0)


def rope_backward(x, weight, eps, positions, inv_freq, dy, interleaved=False, norm=True):
    """(dx, dweight): dweight summed over all rows, None without the norm."""
    x, g = np.asarray(x, np.float64), _turn(dy, positions, inv_freq, interleaved, -1.0)
    if not norm:
        return g, None
    w = np.ones(x.shape[-1]) if weight is None else np.asarray(weight, np.float64)
    var = (x * x).mean(-1, keepdims=True) + eps
    hat = x / np.sqrt(var)
    dw = (g * hat).reshape(-1, x.shape[-1]).sum(0)
    h = g * w
    return (h - hat * (h * hat).mean(-1, keepdims=True)) / np.sqrt(var), dw
