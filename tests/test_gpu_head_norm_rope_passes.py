"""Norms of heads with rotation where a wavefront takes several passes of a token's heads (from 16384 passes in all on): units with a short last one, a last
pass with fewer heads, weights' gradients over passes and tokens, in place; and what few tokens at a time give, one pass a wavefront."""
import numpy as np
import pytest
import torch

import paper_2411_11038_amd as ef
from oracle import attn_oracle as ao

import test_gpu_head_norm_rope as base
from test_gpu_head_norm_rope import E, EPS, by_head, f64, rand, within

pytestmark = pytest.mark.gpu

#        kind, tokens, heads, kv heads, dim, pairs, axes, neighbours, norm; passes of the queries and of the keys
CASES = [(("bf16", 2100, 43, 9, 128, 64, 1, False, True), 6, 2),         # units of 4 and 2 passes; 3 heads and 1 in the last ones
         (("f32", 2100, 43, 9, 128, 64, 1, True, True), 6, 2),
         (("f32", 1900, 33, 25, 80, 36, 3, True, True), 5, 4),           # lanes beside a head's last feature
         (("bf16", 3301, 65, 3, 64, 16, 2, False, True), 5, 1),          # features without a pair
         (("bf16", 2800, 44, 0, 96, 48, 1, False, True), 6, 0),
         (("f32", 2800, 44, 0, 128, 64, 1, False, False), 6, 0)]


def passes(heads, dim):
    lanes = 1
    while lanes * 16 < dim:
        lanes *= 2
    return -(-heads // (64 // lanes))


@pytest.mark.parametrize("n", range(len(CASES)))
def test_several_passes(n):
    args, nq, nk = CASES[n]
    kind, T, dim = args[0], args[1], args[4]
    c = base.Case(*args, apart=8)
    assert (passes(c.heads, dim), passes(c.kv, dim)) == (nq, nk) and T * (nq + nk) > 16384
    u = 2.0 ** -8 if kind == "bf16" else E
    r = ef.head_norm_rope_fwd(c.q, c.heads, k=c.k, **c.how)
    dy = {"q": rand(6, T, c.q.shape[1], kind), "k": rand(7, T, c.k.shape[1], kind) if c.kv else None}
    g = ef.head_norm_rope_bwd(dy["q"], c.q, c.heads, dk=dy["k"], k=c.k, **c.how)
    for name, x, w, heads in c.sides():
        x64, w64, d64 = f64(x), None if w is None else f64(w), f64(dy[name])
        ref = ao.head_norm_rope_fwd(x64, heads, w64, c.norm, EPS, c.t, c.neighbours)
        one = by_head(ao.head_norm_rope_fwd(x64, heads, w64, c.norm, EPS, c.t[:, :0], c.neighbours), heads, lambda v: np.abs(v).max(-1, keepdims=True))
        # as for few tokens: the norm is off by (dim + 12) 2^-24, cosine and sine by 2^-22, of both members of a pair
        within(f64(r[name]), ref, 1.01 * u * np.abs(ref) + ((dim + 12) * E + 8 * E) * 2 * one + 1e-30, name)
        rx, rw = ao.head_norm_rope_bwd(d64, x64, heads, w64, c.norm, EPS, c.t, c.neighbours)
        big = by_head(d64, heads, lambda v: np.abs(v).max(-1, keepdims=True)) * 2
        room = 16 * E * big
        if c.norm:
            rstd = by_head(x64, heads, lambda v: 1.0 / np.sqrt((v * v).mean(-1, keepdims=True) + EPS))
            xhat = by_head(x64 * rstd, heads, lambda v: np.abs(v).max(-1, keepdims=True))
            wmax = 1.0 if w is None else np.abs(w64).max()
            room = (2 * dim + 40) * E * rstd * big * wmax * (1 + xhat * xhat)
            # The weight's gradient, with terms of at most |dn| |xhat|: a term is less than 64 roundings (norm: at most dim / 16 + 4 additions; rotation
            # back of dy, cosine and sine; products).  A lane adds at most 12 passes in fp32, six steps join the lanes and two the
            # wavefronts, the rest is fp64: 64 more.
            dn = np.abs(ao.rotate(d64.reshape(T, heads, -1), -c.t, c.neighbours))
            other = np.abs(d64.reshape(T, heads, -1))
            a, b = ao._pairs(c.t.shape[1], c.neighbours)
            parts = np.maximum(dn, other)
            parts[..., a], parts[..., b] = other[..., a] + other[..., b], other[..., a] + other[..., b]
            terms = (parts * np.abs((x64 * rstd).reshape(T, heads, -1))).sum((0, 1))
            within(f64(g[f"d{name}_weight"]), rw, 128 * E * terms, f"d{name}_weight")
        else:
            assert g["dq_weight"] is None and g["dk_weight"] is None
        within(f64(g["d" + name]), rx, 1.01 * u * np.abs(rx) + room + 1e-30, "d" + name)

    # few tokens at a time: the same arithmetic for every head, bit for bit
    def some(t, rows):
        return None if t is None else t[rows]
    for rows in (slice(0, 700), slice(700, 1400), slice(T - 500, T)):
        how = dict(c.how, positions=c.pos[:, rows].contiguous() if c.axis is not None else c.pos[0, rows].contiguous())
        part = ef.head_norm_rope_fwd(some(c.q, rows), c.heads, k=some(c.k, rows), **how)
        back = ef.head_norm_rope_bwd(some(dy["q"], rows), some(c.q, rows), c.heads, dk=some(dy["k"], rows), k=some(c.k, rows), **how)
        for name, x, w, heads in c.sides():
            assert torch.equal(part[name], r[name][rows]) and torch.equal(back["d" + name], g["d" + name][rows]), name

    # in place, and again
    q, k = c.q.clone(), None if c.k is None else c.k.clone()
    ef.head_norm_rope_fwd(q, c.heads, k=k, out=dict(q=q, k=k) if c.kv else dict(q=q), **c.how)
    dq, dk = dy["q"].clone(), None if dy["k"] is None else dy["k"].clone()
    g2 = ef.head_norm_rope_bwd(dq, c.q, c.heads, dk=dk, k=c.k, out=dict(dq=dq, dk=dk) if c.kv else dict(dq=dq), **c.how)
    for name, a, b in (("q", q, dq), ("k", k, dk)):
        if a is None:
            continue
        assert torch.equal(a, r[name]) and torch.equal(b, g["d" + name])
        assert not c.norm or torch.equal(g2[f"d{name}_weight"], g[f"d{name}_weight"])
