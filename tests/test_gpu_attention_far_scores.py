"""Attention with scores at the end of fp32, and with scores whose product with log2 e passes the size from which the reference is taken from
them first: o and lse against what the scores, exact by choice of the operands, come to in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2411_11038_amd as ef

import attn_checks as ck
from gpu_util import host

pytestmark = pytest.mark.gpu
KINDS = {"bf16": torch.bfloat16, "f32": torch.float32}


def rows_of(n, dim, *columns):
    x = torch.zeros(n, dim, device="cuda")
    for i, c in enumerate(columns):
        x[:, i] = torch.as_tensor(c, dtype=torch.float32, device="cuda")
    return x


def values(n, dim):
    return torch.rand(n, dim, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") + 0.5


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [8, 96, 128])
@pytest.mark.parametrize("q0,k0,scale", [(1.5 * 2.0 ** 64, 2.0 ** 63, 1.0), (1.5 * 2.0 ** 64, -(2.0 ** 63), 1.0), (2.0 ** 63, 2.0 ** 63, 3.0),
                                         (1.5 * 2.0 ** 64, 2.0 ** 63, 3.0), (1.5 * 2.0 ** 64, -(2.0 ** 63), 3.0), (2.0 ** 63, 2.0 ** 63, 1.0)])
def test_scores_at_the_end_of_fp32(kind, dim, q0, k0, scale):
    """all keys have the same score: o is the mean of the values, lse the score (log n is less than its last digit), or an infinity of its sign"""
    n = 150
    q, k, v = (t.to(KINDS[kind]) for t in (rows_of(n, dim, q0), rows_of(n, dim, k0), values(n, dim)))
    r = ef.attention_fwd(q, k, v, 1, scale=scale)
    score = q0 * k0 * scale
    mean = host(v).astype(np.float64).cumsum(0) / np.arange(1, n + 1)[:, None]
    # P is 1 for all keys; a sum of n terms, its quotient, one rounding
    ck.within(host(r["o"]).astype(np.float64), mean, 1.01 * ck.half_step(kind) * mean + (n + 8) * ck.E * 1.5, "o")
    lse = host(r["lse"])[0].astype(np.float64)
    if abs(score) > 3.41e38:
        assert (lse == np.sign(score) * np.inf).all()
    else:
        # log2 e, the product with it, two products with the parts of ln 2: less than four roundings
        ck.within(lse, np.full(n, score), np.full(n, 4 * ck.E * abs(score)), "lse")
    o = ef.attention_decode(q[-1:], k[None], v[None], torch.tensor([n], dtype=torch.int32, device="cuda"), 1, scale=scale)
    ck.within(host(o).astype(np.float64), mean[-1:], 1.01 * ck.half_step(kind) * mean[-1:] + (n + 40) * ck.E * 1.5, "o of the last token alone")


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [8, 128])
@pytest.mark.parametrize("sign", [1, -1])
def test_far_scores_that_share_their_weight(kind, dim, sign):
    """scores 178 (255 or 256) + t, times log2 e short of and past 65536 in the tokens of one tile, t one of seven whole numbers: some keys share
    the weight, the largest of them come late, so that references move between tiles"""
    n, rng = 150, np.random.default_rng(2)
    near = rng.integers(0, 2, n)                             # queries of 255 or 256
    t = rng.integers(-6, 1, n) + np.where(np.arange(n) < 70, -20, 0)
    q, k, v = (x.to(KINDS[kind]) for x in (rows_of(n, dim, 255.0 + near, 1.0), rows_of(n, dim, 178.0 * sign, t.astype(np.float32)), values(n, dim)))
    scores = sign * 178.0 * (255.0 + near)[:, None] + t[None, :]
    assert np.abs(scores[near == 0]).max() * 1.4427 < 65536 < np.abs(scores[near == 1]).min() * 1.4426
    r = ef.attention_fwd(q, k, v, 1, scale=1.0)
    z = np.where(np.tril(np.ones((n, n), bool)), scores, -np.inf)
    top = z.max(1, keepdims=True)
    e = np.exp(z - top)
    ref = (e / e.sum(1, keepdims=True)) @ host(v).astype(np.float64)
    # Short of 65536 all of a row shares the rounding of its reference, half of 2^-8 as an exponent of two.  Two tiles' differ by twice that,
    # once for a reference that moves and once where another token's passes 65536: 2^-7 ln 2 of a probability at most, of the sum as well.
    # Beside it P and o are rounded (bf16), and exponentials and sums of n terms.
    tol = 1.01 * (2 * ck.half_step(kind) + 2 * 2.0 ** -7 * np.log(2.0) + (2 * n + 40) * ck.E) * ref
    ck.within(host(r["o"]).astype(np.float64), ref, tol, "o")
    rl = top[:, 0] + np.log(e.sum(1))
    # the reference's roundings as above, of the sum; those of log2 e, the products with it and with ln 2
    ck.within(host(r["lse"])[0].astype(np.float64), rl, 6 * ck.E * np.abs(rl) + 2 * 2.0 ** -7 * np.log(2.0), "lse")
    o = ef.attention_decode(q[-1:], k[None], v[None], torch.tensor([n], dtype=torch.int32, device="cuda"), 1, scale=1.0)
    ck.within(host(o).astype(np.float64), ref[-1:], tol[-1:], "o of the last token alone")


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [8, 128])
def test_products_beyond_fp32_are_no_number(kind, dim):
    """a token whose product with a key passes fp32 has neither o nor lse: not an infinity, which would pass for a sum; tokens before it have theirs"""
    n = 40
    size = torch.where(torch.arange(n) >= 30, 2.0 ** 65, 1.0)
    q, k, v = (t.to(KINDS[kind]) for t in (rows_of(n, dim, size), rows_of(n, dim, 2.0 ** 64), values(n, dim)))
    r = ef.attention_fwd(q, k, v, 1, scale=1.0)
    o, lse = host(r["o"]), host(r["lse"])[0]
    assert np.isnan(o[30:]).all() and np.isnan(lse[30:]).all()
    mean = host(v).astype(np.float64).cumsum(0) / np.arange(1, n + 1)[:, None]
    ck.within(o[:30].astype(np.float64), mean[:30], (1.01 * ck.half_step(kind) * mean + (n + 8) * ck.E * 1.5)[:30], "o")
    ck.within(lse[:30].astype(np.float64), np.full(30, 2.0 ** 64), np.full(30, 4 * ck.E * 2.0 ** 64), "lse")
