"""CPU oracle of the operators that serve a batch of different requests: rotary embedding with its table, the
4-bit format of the paged cache, attention over what such a cache holds, low-rank adapters.

TEST INFRASTRUCTURE ONLY (same rule as the package).  Plain numpy in fp64, one function per operator; where a format names a
rounding to 32 or 16 bits it stands in its place.  It imports nothing from the GPU package.
"""
from __future__ import annotations

import numpy as np


def rotary_table(rot: int, positions, base: float, factor=1.0, original=0, low=1.0, high=4.0, amplitude=1.0) -> np.ndarray:
    """cos and sin [len(positions), rot / 2, 2] in fp64 (the table holds them rounded to 32 bits)."""
    i = np.arange(rot // 2, dtype=np.float64)
    f = float(base) ** (-2.0 * i / rot)
    if original:
        turns = original * f / (2.0 * np.pi)
        keep = np.clip((turns - low) / (high - low), 0.0, 1.0)
        f = keep * f + (1.0 - keep) * f / factor
    else:
        f = f / factor
    ang = np.asarray(positions, dtype=np.float64)[:, None] * f
    return amplitude * np.stack([np.cos(ang), np.sin(ang)], axis=-1)


def rotate(x_f16, cos_sin, interleaved: bool) -> np.ndarray:
    """Heads x [T, heads, d] with the angles cos_sin [T, rot / 2, 2] of their tokens: the first rot values in pairs, rounded once."""
    x = np.asarray(x_f16, dtype=np.float16).astype(np.float64)
    half = cos_sin.shape[1]
    a, b = (np.arange(0, 2 * half, 2), np.arange(1, 2 * half, 2)) if interleaved else (np.arange(half), np.arange(half, 2 * half))
    c, s = (np.asarray(cos_sin[:, None, :, k], dtype=np.float64) for k in (0, 1))
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y.astype(np.float16)


def q4(x_f16):
    """(codes, steps, offsets) of rows [..., d]: one step and offset per 32 consecutive values, every operation rounded to 32 bits."""
    x = np.asarray(x_f16, dtype=np.float16).astype(np.float32)
    g = x.reshape(*x.shape[:-1], -1, 32)
    lo, hi = g.min(-1, keepdims=True), g.max(-1, keepdims=True)
    step = ((hi - lo) / np.float32(15)).astype(np.float16)
    offset = (lo + np.float32(8) * step.astype(np.float32)).astype(np.float16)
    s = step.astype(np.float32)
    inv = np.where(s > 0, np.float32(1) / np.where(s > 0, s, np.float32(1)), np.float32(0)).astype(np.float32)
    code = np.clip(np.rint((g - offset.astype(np.float32)) * inv) + 8, 0, 15).astype(np.int64)
    return code.reshape(x.shape), step[..., 0], offset[..., 0]


def q4_values(codes, steps, offsets):
    """offset + step (code - 8), fp64, and its two parts' magnitudes added (what roundings of the parts are relative to)."""
    c = (np.asarray(codes).reshape(*codes.shape[:-1], -1, 32) - 8).astype(np.float64)
    s, o = np.asarray(steps, dtype=np.float64)[..., None], np.asarray(offsets, dtype=np.float64)[..., None]
    return (o + s * c).reshape(codes.shape), (np.abs(o) + np.abs(s * c)).reshape(codes.shape)


def attention(q_f16, K, V, V_parts, there=None):
    """Attention of the last S of n positions: q [S, h_q, d]; K, V, V_parts [n, h_kv, d] fp64; there [n] (None: all): positions that are in the cache.
    Returns (out, spread), [S, h_q, d] each: out = softmax(q K^T / sqrt d) V (0 where nothing is seen), spread = sum p V_parts."""
    q = np.asarray(q_f16, dtype=np.float16).astype(np.float64)
    S, h_q, d = q.shape
    n, h_kv = K.shape[:2]
    g = h_q // h_kv
    out, spread = np.zeros((S, h_q, d)), np.zeros((S, h_q, d))
    for s in range(S):
        lim = n - S + s + 1
        if lim <= 0:
            continue
        see = np.arange(lim) if there is None else np.flatnonzero(np.asarray(there)[:lim])
        if see.size == 0:
            continue
        for h in range(h_q):
            k, v = K[see, h // g], V[see, h // g]
            x = k @ q[s, h] / np.sqrt(d)
            p = np.exp(x - x.max())
            p /= p.sum()
            out[s, h] = p @ v
            spread[s, h] = p @ V_parts[see, h // g]
    return out, spread


def adapters(x_f16, ids, a_f16, b_f16, scale, y_f16):
    """(out, spread) [M, N] fp64: y + scale[a] B[a] (A[a] x) per row, and the magnitudes scale |B| |A x| added up."""
    x, a, b, y = (np.asarray(t, dtype=np.float16).astype(np.float64) for t in (x_f16, a_f16, b_f16, y_f16))
    out, spread = y.copy(), np.zeros_like(y)
    for m, i in enumerate(np.asarray(ids)):
        if 0 <= i < a.shape[0]:
            low = a[i] @ x[m]
            out[m] += float(scale[i]) * (b[i] @ low)
            spread[m] = abs(float(scale[i])) * (np.abs(b[i]) @ np.abs(low))
    return out, spread
