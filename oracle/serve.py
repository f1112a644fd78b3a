"""CPU oracle of the serving cache: rows in 8 or 4 bits, attention over them,
a shared prompt's attention joined with the rest, and one head's generation
over such a cache.

TEST INFRASTRUCTURE ONLY, like the rest of this package; it shares no code
with the CUDA path.
"""
from __future__ import annotations

import math

import numpy as np

from . import headkv as O

GROUP = 32


def round_bf16(x) -> np.ndarray:
    """float32 -> the nearest bf16 value (ties to even) as float32."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)
    r = (u + (((u >> np.uint32(16)) & np.uint32(1)) + np.uint32(0x7FFF))) & np.uint32(0xFFFF0000)
    return r.view(np.float32)


def quantise(x, bits: int):
    """Rows x [..., D] -> integer codes [..., D] and scales [..., D / 32]
    (float32 holding bf16 values): of each group of 32 with the largest
    magnitude a, s = bf16(a / M), c = clamp(rint(x / s), -M, M), quotients in
    fp32; s = 0 gives c = 0, a group with a NaN or infinity s = NaN, c = 0."""
    M = np.float32(127 if bits == 8 else 7)
    g = np.asarray(x, dtype=np.float32)
    g = g.reshape(*g.shape[:-1], g.shape[-1] // GROUP, GROUP)
    ok = np.isfinite(g).all(-1)
    a = np.where(ok, np.abs(np.where(ok[..., None], g, 0)).max(-1), 0).astype(np.float32)
    s = round_bf16(a / M).reshape(a.shape)
    safe = np.where(s > 0, s, np.float32(1))[..., None]
    c = np.clip(np.rint(np.where(ok[..., None], g, 0).astype(np.float32) / safe), -M, M)
    c = np.where((s > 0)[..., None], c, 0).astype(np.int64)
    return c.reshape(np.shape(x)), np.where(ok, s, np.float32(np.nan))


def values(codes, scales) -> np.ndarray:
    """What codes and scales stand for, fp64 (exact)."""
    c = np.asarray(codes, dtype=np.float64)
    c = c.reshape(*c.shape[:-1], c.shape[-1] // GROUP, GROUP)
    return (c * np.asarray(scales, dtype=np.float64)[..., None]).reshape(np.shape(codes))


def stored(x, bits: int) -> np.ndarray:
    return values(*quantise(x, bits))


def packed(codes, bits: int) -> np.ndarray:
    """Stored bytes of the codes."""
    c = np.asarray(codes)
    if bits == 8:
        return (c + 128).astype(np.uint8)
    c = (c + 8).astype(np.uint8)
    return c[..., 0::2] | (c[..., 1::2] << 4)


def unpacked(data, bits: int) -> np.ndarray:
    d = np.asarray(data).astype(np.int64)
    if bits == 8:
        return d - 128
    return np.stack([d & 15, d >> 4], -1).reshape(*d.shape[:-1], 2 * d.shape[-1]) - 8


def attention_lse(q, K, V):
    """(softmax(q K^T / sqrt(d)) V, log sum exp), fp64; no keys: (0, -inf)."""
    q, K, V = (np.asarray(x, dtype=np.float64) for x in (q, K, V))
    if K.shape[0] == 0:
        return np.zeros(V.shape[1]), -math.inf
    x = (K @ q) / math.sqrt(q.shape[0])
    m = x.max()
    e = np.exp(x - m)
    return (e @ V) / e.sum(), m + math.log(e.sum())


def run_head_stored(hp: O.HeadParams, q, k, v, bits: int, label: int, record=(),
                    plain_cond: bool = False):
    """Image tokens of one head with the cache in `bits` bits from the grouping
    on (its update still ranks plain keys); plain_cond: the conditioning
    tokens stay plain. Returns ({t: output}, final positions)."""
    C, N, P, E = hp.n_cond, hp.n_image, hp.period, hp.group_at
    ks, vs = stored(k, bits), stored(v, bits)
    if plain_cond:
        ks[:C], vs[:C] = k[:C], v[:C]
    pos = np.arange(C, dtype=np.int64)
    outs, nbuf, compressed = {}, 0, False
    for t in range(N):
        if compressed and nbuf == P:
            pos, nbuf = O.cache_update(pos, label, hp, q, ks.astype(np.float32), t - 1).pos, 0
        pos = np.append(pos, C + t)
        nbuf += compressed
        if t in record:
            K, V = (ks, vs) if compressed else (k, v)
            outs[t] = O.attention(q[t], K[pos], V[pos])
        if t == E - 1:
            pos, nbuf, compressed = O.cache_update(pos, label, hp, q, k, t).pos, 0, True
    return outs, pos
