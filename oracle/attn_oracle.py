"""fp64 NumPy definitions of the operators of an attention block: norms of heads with the position rotation, attention with a window and
first tokens that stay visible, dropout from a counter.  Test infrastructure only: written from the formulas and never imported by the
product path."""
from __future__ import annotations

import math

import numpy as np


# ------------------------------------------------------------------ norms of heads, rotation
def _pairs(freqs, neighbours):
    j = np.arange(freqs)
    return (2 * j, 2 * j + 1) if neighbours else (j, j + freqs)


def angles(positions, inv_freq, axis=None):
    """[T][freqs]; positions [axes][T]"""
    positions, f = np.asarray(positions, np.float64), np.asarray(inv_freq, np.float64)
    axis = np.zeros(f.size, np.int64) if axis is None else np.clip(np.asarray(axis), 0, positions.shape[0] - 1)
    return positions[axis].T * f


def rotate(x, t, neighbours):
    """x [T][heads][dim], angles t [T][freqs]"""
    a, b = _pairs(t.shape[1], neighbours)
    c, s = np.cos(t)[:, None], np.sin(t)[:, None]
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def head_norm_rope_fwd(x, heads, weight, norm, eps, t, neighbours):
    x = np.asarray(x, np.float64).reshape(x.shape[0], heads, -1)
    if norm:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (1.0 if weight is None else weight)
    return rotate(x, t, neighbours).reshape(x.shape[0], -1)


def head_norm_rope_bwd(dy, x, heads, weight, norm, eps, t, neighbours):
    """(dx, dweight)"""
    rows = dy.shape[0]
    d = rotate(np.asarray(dy, np.float64).reshape(rows, heads, -1), -t, neighbours)
    if not norm:
        return d.reshape(rows, -1), None
    x = np.asarray(x, np.float64).reshape(rows, heads, -1)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    xhat = x * r
    g = d * (1.0 if weight is None else weight)
    return (r * (g - xhat * (g * xhat).mean(-1, keepdims=True))).reshape(rows, -1), (d * xhat).sum((0, 1))


# ------------------------------------------------------------------ attention
def seen(nq, nk, causal, window, sinks):
    """bool [nq][nk]: query i is at position i + nk - nq"""
    p, j = np.arange(nq)[:, None] + (nk - nq), np.arange(nk)[None, :]
    out = (j <= p) if causal else np.ones((nq, nk), bool)
    return out & ((abs(p - j) < window) | (j < sinks)) if window else out


def attention_fwd(q, k, v, scale, mask):
    """One sequence and head: (o, lse, P); rows that see nothing: zeros and -inf"""
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    z = np.where(mask, scale * (q @ k.T), -np.inf)
    some = mask.any(1)
    top = np.where(some, z.max(1, initial=-np.inf), 0.0)
    e = np.exp(z - top[:, None])
    total = e.sum(1)
    with np.errstate(divide="ignore"):
        lse = np.where(some, top + np.log(total), -np.inf)
    p = e / np.where(some, total, 1.0)[:, None]
    return p @ v, lse, p


def attention_bwd(do, q, k, v, o, p, scale):
    """One sequence and head, P as attention_fwd has it, o as the backward is given it: (dq, dk, dv, dS)"""
    do, q, k, v, o = (np.asarray(a, np.float64) for a in (do, q, k, v, o))
    ds = p * (do @ v.T - (do * o).sum(1, keepdims=True))
    return scale * ds @ k, scale * ds.T @ q, p.T @ do, ds


# ------------------------------------------------------------------ dropout
def philox4x32(counter, key, rounds=10):
    """counter: four, key: two numbers of 32 bits; the four words"""
    c, k = list(counter), list(key)
    low = 0xFFFFFFFF
    for _ in range(rounds):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & low, (a >> 32) ^ c[3] ^ k[1], a & low]
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    return c


def dropout_mask(rows, cols, p, seed, offset):
    """(bool [rows][cols], factor of what is kept)"""
    least = round(p * 65536)
    low, per_row = 0xFFFFFFFF, -(-cols // 8)
    out = np.zeros((rows, per_row * 8), bool)
    seed, offset = seed % 2 ** 64, offset % 2 ** 64
    for n in range(rows * per_row):
        w = philox4x32((n & low, n >> 32, offset & low, offset >> 32), (seed & low, seed >> 32))
        for j in range(8):
            out[n // per_row, (n % per_row) * 8 + j] = ((w[j // 2] >> (16 * (j % 2))) & 0xFFFF) >= least
    return out[:, :cols], 65536.0 / (65536 - least) if least < 65536 else 0.0


def default_scale(dim):
    return float(np.float32(1.0 / math.sqrt(dim)))
