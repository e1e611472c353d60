"""Float64 oracle of what stands between a layer's linears: norm + rotary + H3 of heads, the paged
4-bit cache, and attention over it and inside packed prompts. Written from the formulas, one loop per
sequence or head; shares nothing with the kernels but their layouts."""

from __future__ import annotations

import math

import numpy as np

from .offq_oracle import sylvester_hadamard


def norm_heads(x, w, eps):
    """RMS norm of x [T, H, D] with weights w [H, D] (None: x itself)."""
    if w is None:
        return x
    return x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * w


def rotary(x, positions, table, interleaved):
    """Rotary positions of the first table.shape[1] channels of x [T, H, D]."""
    y = np.array(x, dtype=np.float64)
    half = table.shape[1] // 2
    for m in range(half):
        a, b = (2 * m, 2 * m + 1) if interleaved else (m, m + half)
        c, s = table[positions, m][:, None], table[positions, half + m][:, None]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def hadamard_heads(x):
    D = x.shape[-1]
    return x @ (sylvester_hadamard(D).astype(np.float64) / math.sqrt(D))


def heads(x, positions=None, table=None, norm=None, eps=0.0, interleaved=False, rotate=False):
    y = norm_heads(np.asarray(x, np.float64), norm, eps)
    if table is not None:
        y = rotary(y, positions, table, interleaved)
    return hadamard_heads(y) if rotate else y


def quantize_heads(y, offset=True):
    """Codes q in -7..7, scales and offsets of heads y, and the residual the codes round."""
    o = y.mean(-1) if offset else np.zeros(y.shape[:-1])
    r = y - o[..., None]
    s = np.abs(r).max(-1) / 7
    q = np.clip(np.rint(np.divide(r, s[..., None], out=np.zeros_like(r), where=s[..., None] > 0)), -7, 7)
    return q.astype(np.int64), s, o, r


def unpack_codes(codes):
    """Signed codes of row-major nibbles, even channel low."""
    c = np.asarray(codes).astype(np.int64)
    return np.stack([c & 15, c >> 4], -1).reshape(*c.shape[:-1], 2 * c.shape[-1]) - 8


def cached(codes, params, pages, at):
    """Values [L, H, D] of the tokens (pages[l], at[l]), and their codes, scales and offsets."""
    q = unpack_codes(codes[pages, :, at])
    p = params[pages, :, at].astype(np.float64)
    return q * p[..., :1] + p[..., 1:], q, p[..., 0], p[..., 1]


def attention(q, k, v, scale, sees):
    """One sequence: q [n, Hq, D], k, v [L, H, D]; query i sees the first sees[i] keys.
    Returns out [n, Hq, D], lse [n, Hq] and the weights [n, Hq, L]."""
    n, Hq, D = q.shape
    L, H = k.shape[0], k.shape[1]
    out, lse, w = np.zeros((n, Hq, D)), np.full((n, Hq), -np.inf), np.zeros((n, Hq, L))
    for h in range(Hq):
        for i in range(n):
            m = max(0, min(L, sees[i]))
            if m == 0:
                continue
            z = k[:m, h * H // Hq] @ q[i, h] * scale
            top = z.max()
            e = np.exp(z - top)
            lse[i, h] = top + np.log(e.sum())
            w[i, h, :m] = e / e.sum()
            out[i, h] = w[i, h, :m] @ v[:m, h * H // Hq]
    return out, lse, w


def attention_masked(q, k, v, scale, seen):
    """The same where query i sees the keys of seen [n, L] (bool)."""
    n, Hq, D = q.shape
    L, H = k.shape[0], k.shape[1]
    out, lse, w = np.zeros((n, Hq, D)), np.full((n, Hq), -np.inf), np.zeros((n, Hq, L))
    some = seen.any(1)
    if not some.any():
        return out, lse, w
    for h in range(Hq):
        z = np.where(seen[some], q[some, h] @ k[:, h * H // Hq].T * scale, -np.inf)
        top = z.max(1, keepdims=True)
        e = np.exp(z - top)
        lse[some, h] = top[:, 0] + np.log(e.sum(1))
        w[some, h] = e / e.sum(1, keepdims=True)
        out[some, h] = w[some, h] @ v[:, h * H // Hq]
    return out, lse, w


def in_window(at, n, L, window, sinks):
    """[n, L]: which tokens queries at positions at .. at + n - 1 see under a sliding window with sinks."""
    p, j = at + np.arange(n)[:, None], np.arange(L)[None]
    return (j <= p) & ((j > p - window) | (j < sinks))
