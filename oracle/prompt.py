"""CPU oracle of what stands around the cache: rotary positions, norms of
heads, and attention of many queries over other states, in fp64.

TEST INFRASTRUCTURE ONLY, like the rest of this package; it shares no code
with the CUDA path.
"""
from __future__ import annotations

import math

import numpy as np


def frequencies(rot_dim, sections, *, joint=False, base=10000.0, scaling="plain", factor=1.0,
                original=1.0, low=1.0, high=32.0) -> np.ndarray:
    """Angles per position of the rot_dim / 2 pairs."""
    f = []
    for n in sections:
        for i in range(n):
            d = rot_dim if joint else 2 * n
            k = len(f) if joint else i
            b = base * factor ** (d / (d - 2)) if scaling == "base" and d > 2 else base
            x = b ** (-2 * k / d)
            if scaling == "linear":
                x /= factor
            if scaling == "parts":
                g = min(1.0, max(0.0, (original * x / (2 * math.pi) - low) / (high - low)))
                x = x * g + x / factor * (1 - g)
            f.append(x)
    return np.array(f)


def rotate(x, angles, layout, amplitude=1.0):
    """Rows x [..., D] by angles [..., rot_dim / 2] (already of the row's token)."""
    y = np.array(x, dtype=np.float64)
    n = angles.shape[-1]
    a, b = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    c, s = amplitude * np.cos(angles), amplitude * np.sin(angles)
    p, q = y[..., a].copy(), y[..., b].copy()
    y[..., a], y[..., b] = p * c - q * s, p * s + q * c
    return y


def angles_of(pos, freq, sections):
    """pos [axes, ...] integers -> angles [..., pairs]; each pair by its axis."""
    axis = np.repeat(np.arange(len(sections)), sections)
    p = np.moveaxis(np.asarray(pos, dtype=np.float64)[axis], 0, -1)
    return p * freq


def norm(x, kind, eps, weight=None, bias=None):
    x = np.asarray(x, dtype=np.float64)
    if kind == "layer":
        x = x - x.mean(-1, keepdims=True)
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    if weight is not None:
        y = y * weight
    return y if bias is None else y + bias


def cross(q, K, V, causal=False):
    """q [n, D] over K, V [m, D] -> (out [n, D], lse [n]); no key: 0, -inf."""
    q, K, V = (np.asarray(x, dtype=np.float64) for x in (q, K, V))
    n, m = len(q), len(K)
    x = q @ K.T / math.sqrt(q.shape[1])
    if causal:
        x[np.arange(m)[None, :] > np.arange(n)[:, None] + m - n] = -math.inf
    top = x.max(-1, keepdims=True, initial=-math.inf)
    e = np.exp(x - np.where(np.isneginf(top), 0, top))
    total = e.sum(-1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = (np.where(np.isneginf(top), 0, top) + np.log(total))[:, 0]
    return e @ V / np.where(total > 0, total, 1), lse
