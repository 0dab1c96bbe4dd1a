"""Plain 64-bit forms of the latent-cache operators for the tests, from their
definitions in include/kamera.h.  numpy only."""

from __future__ import annotations

import math

import numpy as np


def frequencies(theta, rope_dim, kind="none", factor=1.0, original=0.0, low=1.0, high=32.0):
    """Radians a position of every pair."""
    half = rope_dim // 2
    f = np.array([theta ** (-2.0 * j / rope_dim) for j in range(half)])
    if kind == "none":
        return f
    if kind == "linear":
        return f / factor
    if kind == "turns":
        s = (original * f / (2 * math.pi) - low) / (high - low)
    else:
        def J(t):
            return half * math.log(original / (2 * math.pi * t)) / math.log(theta)
        lo, hi = max(math.floor(J(high)), 0), min(math.ceil(J(low)), rope_dim - 1)
        s = 1 - (np.arange(half) - lo) / max(hi - lo, 0.001)
    s = np.clip(s, 0, 1)
    return f * (s + (1 - s) / factor)


def rotate(x, angle, pairing, amplitude=1.0):
    """x [..., rope_dim] by angle [..., rope_dim / 2]; also the sum of the magnitudes that make each element."""
    c, s = np.cos(angle) * amplitude, np.sin(angle) * amplitude
    if pairing == "neox":
        a, b = np.split(x, 2, axis=-1)
    else:
        a, b = x[..., 0::2], x[..., 1::2]
    ra, rb, size = a * c - b * s, a * s + b * c, (np.abs(a) + np.abs(b)) * abs(amplitude)
    if pairing == "neox":
        return np.concatenate([ra, rb], -1), np.concatenate([size, size], -1)
    return np.stack([ra, rb], -1).reshape(x.shape), np.stack([size, size], -1).reshape(x.shape)


def attend_rows(q, k, v, seen, scale):
    """q [n, H, D], k [H or 1, t, D], v [H or 1, t, E], seen [n, t] -> out [n, H, E], the sum of p |v|, lse [n, H], and
    the largest sum |q_j k_j| * |scale|."""
    n, H, _ = q.shape
    out, size, lse = np.zeros((n, H, v.shape[-1])), np.zeros((n, H, v.shape[-1])), np.full((n, H), -math.inf)
    most = 0.0
    for h in range(H):
        kk, vv = k[h % k.shape[0]], v[h % v.shape[0]]
        for i in range(n):
            t = seen[i]
            if not t.any():
                continue
            with np.errstate(invalid="ignore"):
                sc = kk[t] @ q[i, h] * scale
                most = max(most, float((np.abs(kk[t]) @ np.abs(q[i, h])).max()) * abs(scale))
                m = sc.max()
                p = np.exp(sc - m)
                out[i, h] = p @ vv[t] / p.sum()
                size[i, h] = p @ np.abs(vv[t]) / p.sum()
                lse[i, h] = m + math.log(p.sum()) if np.isfinite(m) else math.nan
    return out, size, lse, most


def gather(pool, table, kv, page):
    """Rows [kv, columns] of one request and which of them are in the pool."""
    pos = np.arange(kv)
    pg = table[pos // page] if kv else np.zeros(0, dtype=int)
    ok = (pg >= 0) & (pg < pool.shape[0])
    return pool[np.where(ok, pg, 0), pos % page], ok


def seen_keys(kv, n, causal, window, ok):
    """[n, kv] truth values."""
    pos = np.arange(kv)
    last = kv - n + np.arange(n) if causal else np.full(n, kv - 1)
    seen = ok[None] & (pos[None] <= last[:, None])
    if window:
        seen &= pos[None] > last[:, None] - window
    return seen
