"""The 4-bit KV cache and attention over it in 64 bits, from the definitions in include/ams.h (test infrastructure only).

Nothing here knows the cache's layout: a cache is the list of its sequences' values."""

from __future__ import annotations

import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])  # of the e2m1 codes 0 .. 7 (Sec. 2.2)


def held(x: np.ndarray, scale_group: int) -> np.ndarray:
    """What the cache stands for after rows x, fp16 [..., D], were written: float64, every value one of fp16's."""
    runs = x.astype(np.float64).reshape(*x.shape[:-1], x.shape[-1] // scale_group, scale_group)
    finite = np.isfinite(runs).all(-1, keepdims=True)
    runs = np.where(finite, runs, 0.0)
    s = (np.abs(runs).max(-1, keepdims=True) / 6.0).astype(np.float16).astype(np.float64)
    s = np.minimum(np.where(s == 0, 1.0, s), 10912.0)
    far = np.abs(np.abs(runs)[..., None] / s[..., None] - MAGNITUDES)
    near = far == far.min(-1, keepdims=True)
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), near.argmax(-1))
    y = (MAGNITUDES[code] * s).astype(np.float16).astype(np.float64)
    y = np.where(np.signbit(runs) & (runs != 0), -y, y)
    return np.where(finite, y, np.nan).reshape(x.shape)


def attention(q, k, v, scale, causal=True, window=0):
    """One sequence: q [n, heads, D] at its last n positions over k, v [length, kv_heads, D].

    Returns out [n, heads, D], lse [n, heads] and sum_j p_j |v_j|, which bounds what rounding the weights can do."""
    n, heads, _ = q.shape
    length, kv_heads, _ = k.shape
    position = np.arange(length - n, length)[:, None]
    key = np.arange(length)[None, :]
    seen = np.ones((n, length), dtype=bool) if not causal else key <= position
    if window:
        seen &= key > position - window
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    lse = np.full((n, heads), -np.inf)
    some = seen.any(1)
    if not some.any():
        return out, lse, size
    for h in range(heads):
        kh, vh = k[:, h * kv_heads // heads], v[:, h * kv_heads // heads]
        s = np.where(seen, q[:, h].astype(np.float64) @ kh.T * scale, -np.inf)[some]
        top = s.max(-1, keepdims=True)
        p = np.exp(s - top)
        total = p.sum(-1, keepdims=True)
        out[some, h] = p @ vh / total
        size[some, h] = p @ np.abs(vh) / total
        lse[some, h] = (top + np.log(total))[:, 0]
    return out, lse, size


def scored_attention(q, k, v, scale, causal=True, window=0, softcap=0.0, slopes=None, prefix=0, heads=None):
    """attention with capped scores, a bias by distance (slopes [heads]) and keys below `prefix` that every row with a position sees; of
    q's heads only `heads`, if given.  q may have more rows than there are keys: the first ones have no position."""
    n, all_heads, D = q.shape
    length, kv_heads, _ = k.shape
    position = np.arange(length - n, length)[:, None]
    key = np.arange(length)[None, :]
    seen = np.ones((n, length), dtype=bool)
    if causal:
        seen = (key <= position) & (key > position - (window or length + n))
        seen |= (key < prefix) & (position >= 0)
    heads = range(all_heads) if heads is None else heads
    out, size, lse = np.zeros((n, len(heads), D)), np.zeros((n, len(heads), D)), np.full((n, len(heads)), -np.inf)
    some = seen.any(1)
    if not some.any():
        return out, lse, size
    for i, h in enumerate(heads):
        kh, vh = k[:, h * kv_heads // all_heads], v[:, h * kv_heads // all_heads]
        s = q[:, h].astype(np.float64) @ kh.T * scale
        if softcap:
            s = softcap * np.tanh(s / softcap)
        if slopes is not None:
            s = s - float(slopes[h]) * np.abs(position - key)
        s = np.where(seen, s, -np.inf)[some]
        top = s.max(-1, keepdims=True)
        p = np.exp(s - top)
        total = p.sum(-1, keepdims=True)
        out[some, i] = p @ vh / total
        size[some, i] = p @ np.abs(vh) / total
        lse[some, i] = (top + np.log(total))[:, 0]
    return out, lse, size
