"""fp64 NumPy definitions of the operators between the quantized layers of a language model: 8-bit checkpoints, the activation of
a feed-forward block, layer norm, softmax cross entropy over a vocabulary.  Test infrastructure only: written from the formulas,
one array operation after the other, and never imported by the product path.

Everything is fp64 but the 8-bit codes, which are defined by their fp32 rounding (`ckpt8`)."""
from __future__ import annotations

import math

import numpy as np

GROUP = 128
_erf = np.vectorize(math.erf, otypes=[np.float64])


# ------------------------------------------------------------------ 8-bit checkpoints
def ckpt8(x):
    """(codes int8 [rows][cols], scales fp32 [rows][groups]) of x [rows][cols]: groups of 128 columns, every step in fp32.
    A group with an infinity or a NaN has a scale that is not finite; its codes mean nothing."""
    x = np.asarray(x, np.float32)
    rows, cols = x.shape
    n = -(-cols // GROUP)
    codes = np.zeros((rows, cols), np.int8)
    scales = np.zeros((rows, n), np.float32)
    with np.errstate(all="ignore"):
        for g in range(n):
            part = x[:, g * GROUP:(g + 1) * GROUP]
            s = np.abs(part).max(axis=1) * np.float32(1.0 / 127.0)
            s = np.where(s < np.float32(2.0 ** -126), np.float32(2.0 ** -126), s)
            q = np.rint(part * (np.float32(1.0) / s)[:, None])
            codes[:, g * GROUP:(g + 1) * GROUP] = np.nan_to_num(q, nan=0.0, posinf=127, neginf=-127).astype(np.int8)
            scales[:, g] = s
    return codes, scales


def ckpt8_value(codes, scales):
    """What the codes stand for."""
    cols = codes.shape[1]
    with np.errstate(all="ignore"):
        return codes.astype(np.float64) * np.repeat(scales.astype(np.float64), GROUP, axis=1)[:, :cols]


# ------------------------------------------------------------------ activation
def act(x, kind):
    """(f(x), f'(x))"""
    x = np.asarray(x, np.float64)
    if kind == "gelu":
        phi = 0.5 * (1.0 + _erf(x / math.sqrt(2.0)))
        return x * phi, phi + x * np.exp(-0.5 * x * x) / math.sqrt(2.0 * math.pi)
    s = 1.0 / (1.0 + np.exp(-x))
    return x * s, s * (1.0 + x * (1.0 - s))


def act_fwd(x, kind, up=None):
    y = act(x, kind)[0]
    return y if up is None else y * np.asarray(up, np.float64)


def act_bwd(dy, x, kind, up=None):
    """(dx, dup)"""
    f, slope = act(x, kind)
    dy = np.asarray(dy, np.float64)
    if up is None:
        return dy * slope, None
    return dy * slope * np.asarray(up, np.float64), dy * f


# ------------------------------------------------------------------ layer norm
def layer_norm_fwd(x, weight, bias, eps):
    """(y, mean, rstd)"""
    x = np.asarray(x, np.float64)
    mean = x.mean(axis=1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(axis=1) + eps)
    return (x - mean[:, None]) * rstd[:, None] * weight + bias, mean, rstd


def layer_norm_bwd(dy, x, mean, rstd, weight):
    """(dx, dweight, dbias)"""
    dy, x = np.asarray(dy, np.float64), np.asarray(x, np.float64)
    xhat = (x - mean[:, None]) * rstd[:, None]
    g = dy * weight
    dx = rstd[:, None] * (g - g.mean(axis=1, keepdims=True) - xhat * (g * xhat).mean(axis=1, keepdims=True))
    return dx, (dy * xhat).sum(axis=0), dy.sum(axis=0)


# ------------------------------------------------------------------ cross entropy
def xent(h, w, targets, ignore_index=-100, dloss=None):
    """Per token: (loss, lse, p [T][V], G [T][V]) of the logits h w^T; zero rows for tokens without a class.  dloss [T]: upstream
    gradient of the tokens' losses (None: ones)."""
    h, w = np.asarray(h, np.float64), np.asarray(w, np.float64)
    T, V = h.shape[0], w.shape[0]
    has = (targets != ignore_index) & (targets >= 0) & (targets < V)
    t = np.where(has, targets, 0)
    z = np.zeros((T, V))
    z[has] = h[has] @ w.T
    top = z.max(axis=1)
    lse = np.where(has, top + np.log(np.exp(z - top[:, None]).sum(axis=1)), 0.0)
    loss = np.where(has, lse - z[np.arange(T), t], 0.0)
    p = np.exp(z - lse[:, None]) * has[:, None]
    g = p.copy()
    g[np.arange(T)[has], t[has]] -= 1.0
    if dloss is not None:
        g *= np.where(has, dloss, 0.0)[:, None]
    return loss, lse, p, g
