"""Attention with a window and first tokens that stay visible, forward, backward and for single tokens, against its fp64 definition."""
import numpy as np
import pytest
import torch

import paper_2411_11038_amd as ef
from oracle import attn_oracle as ao

import attn_checks as ck
from gpu_util import host

pytestmark = pytest.mark.gpu
KINDS = {"bf16": torch.bfloat16, "f32": torch.float32}


def rand(seed, rows, cols, kind, std=1.0, apart=0):
    """[rows][cols], rows `apart` elements further than they are long"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(max(rows, 1), cols + apart, generator=g, device="cuda") * std
    return x.to(KINDS[kind])[:rows, :cols]


def offsets(lens):
    return torch.from_numpy(ck.starts(lens)).cuda()


#        causal window sinks
MASKS = [(True, 0, 0), (False, 0, 0), (True, 1, 0), (True, 17, 0), (True, 17, 3), (True, 64, 70), (True, 200, 1), (False, 1, 0), (False, 33, 2), (False, 100, 130)]
# query lengths, key lengths: one token, none, several tiles, fewer keys than queries (rows that see nothing), none of them, a prompt's rest
LENGTHS = [([1], [1]), ([37, 1, 0, 200], [37, 1, 0, 200]), ([65, 5, 3], [64, 0, 300]), ([130, 64], [257, 65])]


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv,dim", [(2, 2, 64), (4, 2, 128), (3, 1, 40), (2, 1, 96), (5, 1, 8)])
@pytest.mark.parametrize("lens", range(len(LENGTHS)))
@pytest.mark.parametrize("mask", range(len(MASKS)))
def test_forward_and_backward(kind, heads, kv, dim, lens, mask):
    causal, window, sinks = MASKS[mask]
    qlens, klens = LENGTHS[lens]
    nq, nk, scale = sum(qlens), sum(klens), ao.default_scale(dim)
    apart = 8 * (mask % 3)
    q, k, v = rand(1, nq, heads * dim, kind, 1.5, apart), rand(2, nk, kv * dim, kind, 1.0, apart), rand(3, nk, kv * dim, kind)
    do = rand(4, nq, heads * dim, kind, 1.0, apart)
    how = dict(kv_heads=kv, q_start=offsets(qlens), k_start=offsets(klens), causal=causal, window=window, sinks=sinks)
    r = ef.attention_fwd(q, k, v, heads, **how)
    ck.check_fwd(r["o"], r["lse"], q, k, v, qlens, klens, heads, kv, scale, causal, window, sinks, kind)
    g = ef.attention_bwd(do, q, k, v, r["o"], r["lse"], heads, **how)
    ck.check_bwd(g["dq"], g["dk"], g["dv"], do, q, k, v, r["o"], r["lse"], qlens, klens, heads, kv, scale, causal, window, sinks, kind)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 128])
def test_even_sequences_and_slices_of_one_tensor(kind, dim):
    """three sequences of 150 tokens without offsets, q, k, v and their gradients slices of stacked tensors: bit for bit as with offsets"""
    heads, kv, n = 4, 2, 450
    x = rand(5, n, (heads + 2 * kv) * dim, kind)
    cut = [heads * dim, (heads + kv) * dim]
    q, k, v = x[:, : cut[0]], x[:, cut[0]: cut[1]], x[:, cut[1]:]
    do = rand(6, n, heads * dim, kind)
    how = dict(kv_heads=kv, window=70, sinks=2)
    r = ef.attention_fwd(q, k, v, heads, sequences=3, **how)
    ck.check_fwd(r["o"], r["lse"], q, k, v, [150] * 3, [150] * 3, heads, kv, ao.default_scale(dim), True, 70, 2, kind)
    dx = torch.full_like(x, 7.0)
    g = ef.attention_bwd(do, q, k, v, r["o"], r["lse"], heads, sequences=3, out=dict(dq=dx[:, : cut[0]], dk=dx[:, cut[0]: cut[1]], dv=dx[:, cut[1]:]), **how)
    start = offsets([150] * 3)
    r2 = ef.attention_fwd(q.contiguous(), k.contiguous(), v.contiguous(), heads, q_start=start, **how)
    g2 = ef.attention_bwd(do, q, k, v, r["o"], r["lse"], heads, q_start=start, k_start=start, **how)
    assert torch.equal(r["o"], r2["o"]) and torch.equal(r["lse"], r2["lse"])
    assert torch.equal(dx, torch.cat((g2["dq"], g2["dk"], g2["dv"]), 1)) and g["dq"].data_ptr() == dx.data_ptr()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_gradient_is_a_difference(kind):
    """the loss sum(o do) of the fp64 definition changes along a direction by the kernel's gradients"""
    heads, kv, dim, n = 2, 1, 64, 90
    q, k, v, do = rand(1, n, 128, kind), rand(2, n, 64, kind), rand(3, n, 64, kind), rand(4, n, 128, kind)
    r = ef.attention_fwd(q, k, v, heads, kv_heads=kv, window=20, sinks=1)
    g = ef.attention_bwd(do, q, k, v, r["o"], r["lse"], heads, kv_heads=kv, window=20, sinks=1)
    mask, rng = ao.seen(n, n, True, 20, 1), np.random.default_rng(0)
    x = [host(t).astype(np.float64) for t in (q, k, v)]
    step = [rng.normal(size=t.shape) for t in x]
    d = host(do).astype(np.float64)

    def loss(e):
        q, k, v = (t + e * s for t, s in zip(x, step))
        return sum((ao.attention_fwd(q[:, 64 * h: 64 * h + 64], k, v, 0.125, mask)[0] * d[:, 64 * h: 64 * h + 64]).sum() for h in range(2))
    slope = (loss(1e-5) - loss(-1e-5)) / 2e-5
    terms = [host(a).astype(np.float64) * s for a, s in zip((g["dq"], g["dk"], g["dv"]), step)]
    # independent errors of a few half steps of each term (their own rounding, those of P, dS and o): four standard deviations
    u = 2.0 ** -8 if kind == "bf16" else 2.0 ** -20
    room = 4 * 4 * u * np.sqrt(sum((t ** 2).sum() for t in terms)) + 1e-6 * abs(slope)
    assert abs(sum(t.sum() for t in terms) - slope) <= room


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_rows_of_no_sequence_stay(kind):
    """rows behind the last sequence (and before the first) hold NaN: they are neither read nor written"""
    heads, dim = 2, 64
    lens, n = [40, 150], 256
    q, k, v, do = (rand(s, n, 128, kind).clone() for s in range(4))
    start = torch.tensor([3, 43, 193], dtype=torch.int32, device="cuda")
    outside = torch.ones(n, dtype=torch.bool, device="cuda")
    outside[3:193] = False
    for t in (q, k, v, do):
        t[outside] = float("nan")
    o, lse = torch.full_like(q, 5.0), torch.full((heads, n), 5.0, device="cuda")
    how = dict(q_start=start, window=30, sinks=2, causal=False)
    ef.attention_fwd(q, k, v, heads, out=dict(o=o, lse=lse), **how)
    grads = {name: torch.full_like(q, 5.0) for name in ("dq", "dk", "dv")}
    ef.attention_bwd(do, q, k, v, o, lse, heads, out=grads, **how)
    for t in (o, *grads.values()):
        assert (t[outside] == 5).all()
    assert (lse[:, outside] == 5).all()
    inner = slice(3, 193)
    a = [t[inner] for t in (q, k, v)]
    ck.check_fwd(o[inner], lse[:, inner], *a, lens, lens, heads, heads, 0.125, False, 30, 2, kind)
    ck.check_bwd(grads["dq"][inner], grads["dk"][inner], grads["dv"][inner], do[inner], *a, o[inner], lse[:, inner], lens, lens, heads, heads, 0.125, False,
                 30, 2, kind)


def test_many_short_sequences():
    """more sequences than a wavefront looks at at a time, empty ones among them"""
    rng = np.random.default_rng(3)
    lens = [int(v) for v in rng.integers(0, 9, 200)] + [0, 0, 140]
    n = sum(lens)
    q, k, v, do = (rand(s, n, 64, "bf16") for s in range(4))
    how = dict(q_start=offsets(lens), causal=False)
    r = ef.attention_fwd(q, k, v, 1, **how)
    ck.check_fwd(r["o"], r["lse"], q, k, v, lens, lens, 1, 1, 0.125, False, 0, 0, "bf16")
    g = ef.attention_bwd(do, q, k, v, r["o"], r["lse"], 1, **how)
    ck.check_bwd(g["dq"], g["dk"], g["dv"], do, q, k, v, r["o"], r["lse"], lens, lens, 1, 1, 0.125, False, 0, 0, "bf16")


@pytest.mark.parametrize("start", [[0, 50, 20, 90], [-5, 30, 30, 4000], [0, 2000000000, -7, 64]])
def test_offsets_that_are_wrong_stay_inside(start):
    """offsets that fall or pass the rows are cut: nothing outside the tensors is touched, and what is written is finite"""
    n = 96
    pool = torch.full((3 * n, 64), 9.0, device="cuda", dtype=torch.bfloat16)
    o = pool[n: 2 * n]
    q, k, v = (rand(s, n, 64, "bf16") for s in range(3))
    s = torch.tensor(start, dtype=torch.int32, device="cuda")
    lse = torch.zeros(1, n, device="cuda")
    o.zero_()
    ef.attention_fwd(q, k, v, 1, q_start=s, k_start=s, out=dict(o=o, lse=lse))
    grads = {name: torch.zeros_like(q) for name in ("dq", "dk", "dv")}
    ef.attention_bwd(q, q, k, v, o, lse, 1, q_start=s, k_start=s, out=grads)
    assert (pool[:n] == 9).all() and (pool[2 * n:] == 9).all()
    assert all(torch.isfinite(t).all() for t in (o, *grads.values()))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_large_scores(kind):
    """scores of some hundreds: one key takes nearly all, nothing overflows"""
    n, dim = 70, 128
    q, k, v, do = rand(1, n, dim, kind, 30.0), rand(2, n, dim, kind, 10.0), rand(3, n, dim, kind), rand(4, n, dim, kind)
    r = ef.attention_fwd(q, k, v, 1)
    ck.check_fwd(r["o"], r["lse"], q, k, v, [n], [n], 1, 1, ao.default_scale(dim), True, 0, 0, kind)
    g = ef.attention_bwd(do, q, k, v, r["o"], r["lse"], 1)
    ck.check_bwd(g["dq"], g["dk"], g["dv"], do, q, k, v, r["o"], r["lse"], [n], [n], 1, 1, ao.default_scale(dim), True, 0, 0, kind)


def test_values_that_are_not_finite_stay_in_their_sequence_and_head():
    heads, dim, lens = 2, 64, [50, 60]
    q, k, v = (rand(s, 110, 128, "bf16").clone() for s in range(3))
    clean = ef.attention_fwd(q, k, v, heads, q_start=offsets(lens))
    v[20, 3], k[70, 64] = float("inf"), float("nan")         # sequence 0 head 0, sequence 1 head 1
    r = ef.attention_fwd(q, k, v, heads, q_start=offsets(lens))
    for rows, cols in ((slice(0, 50), slice(64, 128)), (slice(50, 110), slice(0, 64))):
        assert torch.equal(r["o"][rows, cols], clean["o"][rows, cols])
    assert not torch.isfinite(r["o"][20:50, 3]).any() and torch.isnan(r["o"][70:110, 64:]).all()


def test_large_window_is_none():
    q, k, v = (rand(s, 100, 64, "bf16") for s in range(3))
    a = ef.attention_fwd(q, k, v, 1)
    for w in (100, 2 ** 28, 2 ** 40):
        b = ef.attention_fwd(q, k, v, 1, window=w, sinks=2 ** 40 if w > 100 else 0)
        assert torch.equal(a["o"], b["o"]) and torch.equal(a["lse"], b["lse"])


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv,dim", [(1, 1, 64), (8, 2, 128), (40, 1, 64), (6, 3, 40), (16, 1, 128)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (50, 4), (300, 40)])
def test_decode(kind, heads, kv, dim, window, sinks):
    cap = 1000
    lens = [1, 0, 33, 1000, 517, 64]
    n = len(lens)
    q = rand(1, n, heads * dim, kind, 1.5, 16)
    k, v = (rand(s, n * cap, kv * dim, kind, 1.0, 8 * s).clone().view(n, cap, -1) for s in (2, 3))
    for s, m in enumerate(lens):
        k[s, m:] = float("nan")                              # a cache holds anything there
        v[s, m:] = float("inf")
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    o = ef.attention_decode(q, k, v, lengths, heads, kv_heads=kv, window=window, sinks=sinks)
    for s, m in enumerate(lens):
        if m == 0:
            assert (o[s] == 0).all()
            continue
        _, rl, _ = ao.attention_fwd(np.zeros((1, dim)), np.zeros((m, dim)), np.zeros((m, dim)), 1.0, np.ones((1, m), bool))
        one = torch.zeros(heads, 1, device="cuda")
        Q, K, V = ck.heads_of(q[s: s + 1], heads), ck.heads_of(k[s, :m], kv), ck.heads_of(v[s, :m], kv)
        u, O = ck.half_step(kind), ck.heads_of(o[s: s + 1], heads)
        mask = ao.seen(1, m, True, window, sinks)
        for h in range(heads):
            g = h * kv // heads
            ref, lse, p = ao.attention_fwd(Q[h], K[g], V[g], ao.default_scale(dim), mask)
            size = ao.default_scale(dim) * (np.abs(Q[h]) @ np.abs(K[g]).T)
            eta = np.where(mask, ck._spread(size, lse, dim), 0.0)
            # partial sums are put together with two more factors of exponentials each
            tol = 1.01 * u * np.abs(ref) + 1.01 * (p * (u + eta + eta.max() + (m + 8 + 32) * ck.E)) @ np.abs(V[g]) + 1e-30
            ck.within(O[h], ref, tol, f"sequence {s} head {h}")
            if kind == "bf16":
                ck.near(O[h], ref, u * np.sqrt(ref ** 2 + p ** 2 @ V[g] ** 2), (p * (eta + eta.max() + (m + 8 + 32) * ck.E)) @ np.abs(V[g]),
                        f"sequence {s} head {h}")


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 128])
def test_every_key_has_its_weight(kind, dim):
    """values that say which key they belong to, at every length of a last tile of 32, and at windows that begin anywhere in one"""
    for n, window in [(64 + i, 0) for i in range(33)] + [(200, 100 + i) for i in range(33)]:
        q, k = rand(n, 1, dim, kind, 2.0), rand(n + 1, n, dim, kind)
        lo = n - window if window else 0
        p = ao.attention_fwd(host(q), host(k), np.zeros((n, 1)), ao.default_scale(dim), ao.seen(1, n, True, window, 0))[2][0]
        got = np.zeros(n)
        for b in range(0, n, dim):
            v = torch.zeros(n, dim, device="cuda", dtype=KINDS[kind])
            m = min(dim, n - b)
            v[torch.arange(b, b + m), torch.arange(m)] = 1
            o = ef.attention_decode(q, k[None], v[None], torch.tensor([n], dtype=torch.int32, device="cuda"), 1, window=window)
            got[b: b + m] = host(o)[0, :m]
        # P and the result are rounded, the score is off by (dim + 8) 2^-24 of at most 40
        u = 2 * ck.half_step(kind) + 2.0 ** -15
        assert (got[:lo] == 0).all() and (np.abs(got - p) <= u * p).all(), (n, window, np.argmax(np.abs(got - p) / np.maximum(p, 1e-30)))


def test_decode_cache_strides_and_one_sequence():
    """caches laid out [capacity][sequences], one that all sequences share, and lengths beyond the capacity"""
    q = rand(1, 3, 256, "bf16")
    k, v = (rand(s, 300 * 3, 128, "bf16").view(300, 3, 128).transpose(0, 1) for s in (2, 3))
    lengths = torch.tensor([300, 7, 200], dtype=torch.int32, device="cuda")
    a = ef.attention_decode(q, k, v, lengths, 4, kv_heads=2)
    b = ef.attention_decode(q, k.contiguous(), v.contiguous(), lengths * torch.tensor([100, 1, 1], dtype=torch.int32, device="cuda"), 4, kv_heads=2)
    assert torch.equal(a, b)
    one = [t[1:2].expand(3, 300, 128) for t in (k, v)]
    a = ef.attention_decode(q, *one, lengths, 4, kv_heads=2)
    assert torch.equal(a, ef.attention_decode(q, *(t.contiguous() for t in one), lengths, 4, kv_heads=2))
    assert torch.equal(ef.attention_decode(q[2:], k[2:], v[2:], lengths[2:], 4, kv_heads=2), b[2:])


@pytest.mark.parametrize("scale", [1e-39, 1e-38, 1e-20, 1e30])
def test_extreme_scales(scale):
    """so small that no score reaches the step by which the reference score moves, and so large that one key takes all"""
    n = 100
    q, k, v = rand(1, n, 64, "f32"), rand(2, n, 64, "f32"), rand(3, n, 64, "f32")
    r = ef.attention_fwd(q, k, v, 1, scale=scale)
    if scale < 1:
        mean = v.double().cumsum(0) / torch.arange(1, n + 1, device="cuda")[:, None]
        assert (r["o"].double() - mean).abs().max() < (n + 8) * ck.E * v.abs().max()
        assert (r["lse"][0].double() - torch.arange(1, n + 1, device="cuda").double().log()).abs().max() < 1e-6
    else:
        best = (q.double() @ k.double().t()).masked_fill(torch.ones(n, n, device="cuda").triu(1).bool(), -1e300).argmax(1)
        assert torch.equal(r["o"], v[best])
        one = ef.attention_decode(q[-1:], k[None], v[None], torch.tensor([n], dtype=torch.int32, device="cuda"), 1, scale=scale)
        assert torch.equal(one, v[best[-1:]])


def test_decode_is_the_last_row_of_the_forward():
    heads, kv, dim, n = 8, 2, 128, 777
    q, k, v = rand(1, n, heads * dim, "f32"), rand(2, n, kv * dim, "f32"), rand(3, n, kv * dim, "f32")
    for window, sinks in ((0, 0), (100, 5)):
        a = ef.attention_fwd(q, k, v, heads, kv_heads=kv, window=window, sinks=sinks)["o"][-1:]
        b = ef.attention_decode(q[-1:], k[None], v[None], torch.tensor([n], dtype=torch.int32, device="cuda"), heads, kv_heads=kv, window=window, sinks=sinks)
        assert (a - b).abs().max() <= 1e-5 * v.abs().max()   # both within (777 + 136) 2^-24 and the scores' 2^-16 of it


def test_decode_past_32_bits():
    """a cache of more than 2^31 elements: the last sequence's keys lie behind that"""
    n, cap, cols = 3, 1 << 20, 1024
    k = torch.zeros(n, cap, cols, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros(n, cap, cols, dtype=torch.bfloat16, device="cuda")
    k[2, -40:] = rand(2, 40, cols, "bf16")
    v[2, -40:] = rand(3, 40, cols, "bf16")
    q = rand(1, n, cols, "bf16")
    lengths = torch.full((n,), cap, dtype=torch.int32, device="cuda")
    o = ef.attention_decode(q, k, v, lengths, 8, window=40)
    small = ef.attention_decode(q[2:], k[2:, -40:].contiguous(), v[2:, -40:].contiguous(), torch.tensor([40], dtype=torch.int32, device="cuda"), 8)
    assert (o[:2] == 0).all() and (o[2:].float() - small.float()).abs().max() <= 2 ** -7 * v.abs().max().float()     # tiles cut elsewhere
    del k, v


def test_refusals():
    q, k, v = (rand(s, 64, 128, "bf16") for s in range(3))
    ok = ef.attention_fwd(q, k, v, 2)
    length = torch.tensor([64], dtype=torch.int32, device="cuda")
    for bad in (dict(heads=3), dict(heads=2, kv_heads=1), dict(heads=0), dict(heads=2, k_start=length), dict(heads=2, out=dict(lse=torch.zeros(2, 63, device="cuda")))):
        with pytest.raises(ValueError):
            ef.attention_fwd(q, k, v, **bad)
    for t in ((q.float(), k, v), (q, k, v.float()), (q.half(), k.half(), v.half())):
        with pytest.raises(TypeError):
            ef.attention_fwd(*t, 2)
    with pytest.raises(ValueError):
        ef.attention_fwd(q.cpu(), k, v, 2)
    with pytest.raises(ValueError):
        ef.attention_fwd(q, k[:63], v, 2)
    with pytest.raises(ef.EfqatError):
        ef.attention_fwd(q, k, v, 2, sequences=3)
    with pytest.raises(ef.EfqatError):
        ef.attention_fwd(q, k, v, 2, window=-1)
    with pytest.raises(ef.EfqatError):
        ef.attention_fwd(rand(1, 64, 128, "bf16", 1.0, 4), k, v, 2)      # rows 264 bytes apart
    with pytest.raises(TypeError):
        ef.attention_fwd(q, k, v, 2, q_start=torch.tensor([0, 64], device="cuda"))
    with pytest.raises(ValueError):
        ef.attention_bwd(q, q, k, v, ok["o"], ok["lse"][:1], 2)
    with pytest.raises(ef.EfqatError):
        ef.attention_bwd(q, q, k, v, ok["o"], ok["lse"], 2, ws=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        ef.attention_decode(q[:1], k, v, length, 2)
    with pytest.raises(TypeError):
        ef.attention_decode(q[:1], k[None], v[None], length.long(), 2)
    with pytest.raises(ValueError):
        ef.attention_decode(q[:2], k[None], v[None], length, 2)
