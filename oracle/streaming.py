"""Streaming operators in 64 bits: rotary positions, the append to a paged cache, and softmax
attention of packed sequences with the token- or block-causal mask."""
from __future__ import annotations

import numpy as np


def rope_angles(pos, inv_freq):
    """[T][rot / 2] angles in radians of positions pos [T] and frequencies inv_freq [rot / 2]."""
    return np.asarray(pos, np.float64)[:, None] * np.asarray(inv_freq, np.float64)[None, :]


def rope(x, angles, interleaved=False, scale=1.0):
    """x [T][heads][d] with its first 2 x angles.shape[1] channels rotated in pairs: (i, i + rot / 2),
    or (2 i, 2 i + 1) when interleaved; (a, b) -> scale (a cos - b sin, b cos + a sin)."""
    x = np.array(x, np.float64)
    half = angles.shape[1]
    a_at = slice(0, 2 * half, 2) if interleaved else slice(0, half)
    b_at = slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half)
    a, b = x[..., a_at].copy(), x[..., b_at].copy()
    c, s = scale * np.cos(angles)[:, None], scale * np.sin(angles)[:, None]
    x[..., a_at] = a * c - b * s
    x[..., b_at] = b * c + a * s
    return x


def row_limits(n, L, block):
    """lim(i) of the n new tokens of a sequence of L tokens: row i sees the keys j < lim(i)."""
    i = np.arange(n)
    if block == 0:
        return np.full(n, L)
    return L - n + np.minimum(n, (i // block + 1) * block)


def seq_attention(q, k, v, lim, scale):
    """One sequence: q [n][Hq][d], k, v [L][Hkv][d], lim [n].  Returns (out [n][Hq][d], lse [n][Hq],
    spread [n][Hq][d]), spread = sum_j p_j |v_j| (what a relative error of the p_j is measured by).
    Keys a row does not see are left out of its sums altogether."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    n, Hq, d = q.shape
    g = Hq // k.shape[1]
    out, lse, spread = np.zeros((n, Hq, d)), np.full((n, Hq), -np.inf), np.zeros((n, Hq, d))
    lim = np.asarray(lim)
    for value in np.unique(lim):
        if value <= 0:
            continue
        rows = np.flatnonzero(lim == value)
        kk, vv = k[:value], v[:value]
        for h in range(Hq):
            with np.errstate(invalid="ignore", over="ignore"):
                s = scale * (q[rows, h] @ kk[:, h // g].T)
                m = s.max(-1, keepdims=True)
                p = np.exp(s - m)
                l = p.sum(-1, keepdims=True)
                out[rows, h] = p @ vv[:, h // g] / l
                spread[rows, h] = p @ np.abs(vv[:, h // g]) / l
                lse[rows, h] = (m + np.log(l))[:, 0]
    return out, lse, spread
