"""Norms of queries and keys for each head with the position rotation, forward and backward, against their fp64 definition."""
import numpy as np
import pytest
import torch

import paper_2411_11038_amd as ef
from oracle import attn_oracle as ao

from gpu_util import host

pytestmark = pytest.mark.gpu
KINDS = {"bf16": torch.bfloat16, "f32": torch.float32}
E, EPS = 2.0 ** -24, 1e-6


def rand(seed, rows, cols, kind="f32", std=1.0, mean=0.0, apart=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(rows, cols + apart, generator=g, device="cuda") * std + mean).to(KINDS[kind])[:, :cols]


def f64(t):
    return host(t).astype(np.float64)


def within(got, ref, tol, what):
    assert got.shape == ref.shape and np.isfinite(got).all(), what
    bad = np.abs(got - ref) > tol
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.abs(got - ref)[bad].max():.3e} where {tol[bad].min():.3e} is allowed"


def by_head(x, heads, fn):
    """fn of every head's row, spread over its features"""
    r = x.reshape(x.shape[0], heads, -1)
    return np.broadcast_to(fn(r), r.shape).reshape(x.shape)


class Case:
    def __init__(self, kind, T, heads, kv, dim, freqs, axes, neighbours, norm, weights=True, apart=0):
        self.kind, self.heads, self.kv, self.neighbours = kind, heads, kv, neighbours
        self.q, self.k = rand(1, T, heads * dim, kind, 1.5, 0.2, apart), (rand(2, T, kv * dim, kind, 0.5, 0.0, 2 * apart) if kv else None)
        self.wq, self.wk = (rand(3, 1, dim, "f32", 0.2, 1.0)[0], rand(4, 1, dim, "f32", 0.2, 1.0)[0]) if weights and norm else (None, None)
        g = torch.Generator(device="cuda").manual_seed(5)
        self.pos = torch.randint(-100, 100000, (axes, T), generator=g, device="cuda", dtype=torch.int32)
        self.f = (10000.0 ** (-torch.arange(freqs, device="cuda") / max(freqs, 1))).float() if freqs else None
        self.axis = torch.randint(-1, axes + 1, (freqs,), generator=g, device="cuda", dtype=torch.int32) if axes > 1 and freqs else None
        self.how = dict(kv_heads=kv, q_weight=self.wq, k_weight=self.wk if kv else None, norm=norm, eps=EPS, neighbours=neighbours)
        if freqs:
            self.how.update(positions=self.pos if axes > 1 else self.pos[0], inv_freq=self.f, axis=self.axis)
        self.norm = norm
        self.t = ao.angles(self.pos.cpu().numpy(), np.zeros(0) if self.f is None else f64(self.f), None if self.axis is None else self.axis.cpu().numpy())

    def sides(self):
        yield "q", self.q, self.wq, self.heads
        if self.kv:
            yield "k", self.k, self.wk, self.kv


CASES = [("bf16", 5, 8, 2, 128, 64, 1, False, True), ("bf16", 33, 4, 4, 64, 32, 3, True, True), ("f32", 7, 3, 1, 80, 36, 2, True, True),
         ("f32", 130, 2, 2, 128, 32, 1, False, True), ("bf16", 3, 5, 0, 256, 128, 1, False, True), ("f32", 1, 1, 1, 8, 4, 1, True, False),
         ("bf16", 70, 40, 8, 128, 64, 1, False, False), ("f32", 9, 3, 2, 33, 11, 2, False, True), ("bf16", 21, 2, 1, 200, 37, 4, True, True),
         ("bf16", 64, 6, 3, 96, 12, 1, False, True), ("f32", 40, 4, 2, 64, 0, 1, False, True), ("f32", 6, 7, 3, 255, 1, 1, True, True),
         ("bf16", 5000, 3, 1, 64, 32, 1, False, True), ("f32", 2000, 12, 12, 40, 20, 3, True, True), ("f32", 4, 2, 2, 16, 8, 1, False, False)]


@pytest.mark.parametrize("n", range(len(CASES)))
@pytest.mark.parametrize("apart", [0, 3])
def test_forward_and_backward(n, apart):
    c = Case(*CASES[n], apart=apart)
    kind, T = CASES[n][0], CASES[n][1]
    u = 2.0 ** -8 if kind == "bf16" else E
    r = ef.head_norm_rope_fwd(c.q, c.heads, k=c.k, **c.how)
    assert c.kv or r["k"] is None
    dy = {"q": rand(6, T, c.q.shape[1], kind, 1.0, 0.0, apart), "k": rand(7, T, c.k.shape[1], kind) if c.kv else None}
    g = ef.head_norm_rope_bwd(dy["q"], c.q, c.heads, dk=dy["k"], k=c.k, **c.how)
    for name, x, w, heads in c.sides():
        x64, w64 = f64(x), None if w is None else f64(w)
        dim = x64.shape[1] // heads
        ref = ao.head_norm_rope_fwd(x64, heads, w64, c.norm, EPS, c.t, c.neighbours)
        # fp32 throughout, rounded once: the norm is off by (dim + 12) 2^-24, cosine and sine by 2^-22, of both members of a pair
        one = by_head(ao.head_norm_rope_fwd(x64, heads, w64, c.norm, EPS, c.t[:, :0], c.neighbours), heads, lambda v: np.abs(v).max(-1, keepdims=True))
        within(f64(r[name]), ref, 1.01 * u * np.abs(ref) + ((dim + 12) * E + 8 * E) * 2 * one + 1e-30, name)
        d64 = f64(dy[name])
        rx, rw = ao.head_norm_rope_bwd(d64, x64, heads, w64, c.norm, EPS, c.t, c.neighbours)
        big = by_head(d64, heads, lambda v: np.abs(v).max(-1, keepdims=True)) * 2
        if c.norm:
            rstd = by_head(x64, heads, lambda v: 1.0 / np.sqrt((v * v).mean(-1, keepdims=True) + EPS))
            xhat = by_head(x64 * rstd, heads, lambda v: np.abs(v).max(-1, keepdims=True))
            wmax = 1.0 if w is None else np.abs(w64).max()
            # g and xhat mean(g xhat), |mean(g xhat)| at most max|g| max|xhat|, each off by (2 dim + 40) 2^-24
            room = (2 * dim + 40) * E * rstd * big * wmax * (1 + xhat * xhat)
            # the weight's gradient: terms off by (dim + 40) 2^-24, partial sums of at most T heads terms in fp32
            tw = (dim + 40 + T * heads) * E * 2 * (big * xhat).reshape(-1, dim).sum(0)
            within(f64(g[f"d{name}_weight"]), rw, 1.01 * E * np.abs(rw) + tw, f"d{name}_weight")
        else:
            room = 16 * E * big
            assert g["dq_weight"] is None and g["dk_weight"] is None
        within(f64(g["d" + name]), rx, 1.01 * u * np.abs(rx) + room + 1e-30, "d" + name)


@pytest.mark.parametrize("dim,freqs,neighbours", [(64, 32, False), (64, 20, True), (36, 18, False)])
def test_in_place(dim, freqs, neighbours):
    """the queries and keys of a stacked product turned where they lie, and their gradients"""
    T, heads, kv = 50, 4, 2
    x = rand(1, T, (heads + 2 * kv) * dim, "bf16")
    cut = [heads * dim, (heads + kv) * dim]
    w = rand(2, 1, dim)[0]
    how = dict(kv_heads=kv, q_weight=w, k_weight=w, positions=torch.arange(T, device="cuda", dtype=torch.int32),
               inv_freq=torch.rand(freqs, device="cuda"), neighbours=neighbours)

    def sides(t):
        return t[:, : cut[0]], t[:, cut[0]: cut[1]]
    q, k = sides(x)
    r = ef.head_norm_rope_fwd(q, heads, k=k, **how)
    y = x.clone()
    a, b = sides(y)
    ef.head_norm_rope_fwd(a, heads, k=b, out=dict(q=a, k=b), **how)
    assert torch.equal(a, r["q"]) and torch.equal(b, r["k"]) and torch.equal(y[:, cut[1]:], x[:, cut[1]:])
    dy = rand(3, T, x.shape[1], "bf16")
    dq, dk = sides(dy)
    g = ef.head_norm_rope_bwd(dq, q, heads, dk=dk, k=k, **how)
    d = dy.clone()
    a, b = sides(d)
    g2 = ef.head_norm_rope_bwd(a, q, heads, dk=b, k=k, out=dict(dq=a, dk=b), **how)
    assert torch.equal(a, g["dq"]) and torch.equal(b, g["dk"]) and torch.equal(d[:, cut[1]:], dy[:, cut[1]:])
    assert torch.equal(g["dq_weight"], g2["dq_weight"]) and torch.equal(g["dk_weight"], g2["dk_weight"])


@pytest.mark.parametrize("dim", [64, 33])
def test_far_positions(dim):
    """angles of positions up to 2^31: the turn is taken from the exact product"""
    pos = torch.tensor([2 ** 31 - 1, -2 ** 31, 16777217, 123456789], dtype=torch.int32, device="cuda")
    f = torch.tensor([1.0, 0.7071067811865476, 1e-4, 3.1], device="cuda") if dim == 33 else torch.rand(8, device="cuda")
    x = rand(1, 4, dim)
    y = f64(ef.head_norm_rope_fwd(x, 1, norm=False, positions=pos, inv_freq=f)["q"])
    ref = ao.head_norm_rope_fwd(f64(x), 1, None, False, 0.0, ao.angles(pos.cpu().numpy()[None], f64(f)), False)
    # three roundings of 2^-53 of at most 2^31 3.1 radians, both here and in the definition's angle: 2^-18.4 in all, beside 2^-21 of fp32
    assert np.abs(y - ref).max() <= 2 * (2.0 ** -18 + 2.0 ** -21) * np.abs(f64(x)).max()


def test_what_has_no_pair_is_untouched_by_infinities():
    for dim, freqs, neighbours in ((64, 8, False), (64, 5, True), (36, 5, False)):
        x = rand(1, 3, dim).clone()
        x[:, 2 * freqs + 1] = float("inf")
        y = ef.head_norm_rope_fwd(x, 1, norm=False, positions=torch.arange(3, device="cuda", dtype=torch.int32),
                                  inv_freq=torch.ones(freqs, device="cuda"), neighbours=neighbours)["q"]
        assert torch.equal(y[:, 2 * freqs:], x[:, 2 * freqs:]) and torch.isfinite(y[:, : 2 * freqs]).all()


def test_zero_heads_and_large_values():
    x = torch.zeros(2, 64, device="cuda")
    x[1] = 1e30
    y = ef.head_norm_rope_fwd(x, 1)["q"]
    assert (y == 0).all()                                   # nothing over eps; squares that leave fp32


@pytest.mark.parametrize("dim", [64, 40, 33])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_norm_without_eps(kind, dim):
    """eps 0: heads that fill a part of a wavefront; what lies beside them is no head whose norm is 0 / 0"""
    T, heads, kv = 5, 3, 1
    q, k, dq, dk = rand(1, T, heads * dim, kind, 1.0, 0.5), rand(2, T, dim, kind), rand(3, T, heads * dim, kind), rand(4, T, dim, kind)
    w = rand(5, 1, dim, "f32", 0.2, 1.0)[0]
    g = ef.head_norm_rope_bwd(dq, q, heads, dk=dk, k=k, kv_heads=kv, q_weight=w, k_weight=w, eps=0.0)
    for name, x, dy, n in (("q", q, dq, heads), ("k", k, dk, kv)):
        x, dy = f64(x).reshape(T, n, dim), f64(dy).reshape(T, n, dim)
        terms = dy * x / np.sqrt((x * x).mean(-1, keepdims=True))
        # a term: the norm's sum of squares (dim / 16 + 4 additions of at most that many roundings each, halved by the root), root, reciprocal
        # and two products: less than 64 roundings of 2^-24; sums of the terms T * heads more, all of the terms' sizes
        within(f64(g[f"d{name}_weight"]), terms.sum((0, 1)), (64 + T * n) * E * np.abs(terms).sum((0, 1)) + 1e-30, f"d{name}_weight")
        assert torch.isfinite(g["d" + name].float()).all()


def test_same_results_each_time():
    q, k, d = rand(1, 3000, 512, "bf16"), rand(2, 3000, 128, "bf16"), rand(3, 3000, 640, "bf16")
    a, b = (ef.head_norm_rope_bwd(d[:, :512], q, 4, dk=d[:, 512:], k=k, kv_heads=1) for _ in range(2))
    assert all(torch.equal(a[n], b[n]) for n in a)


def test_refusals():
    q, k = rand(1, 4, 128), rand(2, 4, 64)
    pos, f = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.ones(8, device="cuda")
    for bad in (dict(heads=3), dict(heads=2, k=k), dict(heads=2, k=k, kv_heads=2), dict(heads=2, positions=pos), dict(heads=2, inv_freq=f),
                dict(heads=2, positions=pos[:3], inv_freq=f), dict(heads=2, q_weight=torch.ones(128, device="cuda")),
                dict(heads=2, out=dict(q=k))):
        with pytest.raises(ValueError):
            ef.head_norm_rope_fwd(q, **bad)
    for bad in (dict(positions=pos.long(), inv_freq=f), dict(positions=pos, inv_freq=f.double()), dict(k=k.bfloat16(), kv_heads=1)):
        with pytest.raises(TypeError):
            ef.head_norm_rope_fwd(q, 2, **bad)
    with pytest.raises(ef.EfqatError):
        ef.head_norm_rope_fwd(q, 2, positions=pos, inv_freq=torch.ones(33, device="cuda"))
    with pytest.raises(ef.EfqatError):
        ef.head_norm_rope_fwd(q, 2, positions=pos.expand(2, 4).contiguous(), inv_freq=f)      # two axes, none named
    with pytest.raises(ValueError):
        ef.head_norm_rope_bwd(q, None, 2)
    with pytest.raises(ef.EfqatError):
        ef.head_norm_rope_bwd(q, q, 2, ws=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        ef.head_norm_rope_fwd(q.cpu(), 2)
