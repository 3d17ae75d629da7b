"""Attention where its work is cut: keys with sinks whose far queries are the work of blocks of their own, tiles of keys in parts and whole; the
same results each time, in captured graphs and on other streams."""
import numpy as np
import pytest
import torch

import paper_2411_11038_amd as ef
from oracle import attn_oracle as ao

import attn_checks as ck

pytestmark = pytest.mark.gpu
KINDS = {"bf16": torch.bfloat16, "f32": torch.float32}


def rand(seed, rows, cols, kind, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(rows, cols, generator=g, device="cuda") * std).to(KINDS[kind])


def run(kind, qlens, klens, heads, kv, dim, causal, window, sinks, check=True):
    nq, nk = sum(qlens), sum(klens)
    q, k, v, do = rand(1, nq, heads * dim, kind, 1.5), rand(2, nk, kv * dim, kind), rand(3, nk, kv * dim, kind), rand(4, nq, heads * dim, kind)
    how = dict(kv_heads=kv, q_start=torch.from_numpy(ck.starts(qlens)).cuda(), k_start=torch.from_numpy(ck.starts(klens)).cuda(), causal=causal,
               window=window, sinks=sinks)
    r = ef.attention_fwd(q, k, v, heads, **how)
    g = ef.attention_bwd(do, q, k, v, r["o"], r["lse"], heads, **how)
    if check:
        args = (qlens, klens, heads, kv, ao.default_scale(dim), causal, window, sinks, kind)
        ck.check_fwd(r["o"], r["lse"], q, k, v, *args)
        ck.check_bwd(g["dq"], g["dk"], g["dv"], do, q, k, v, r["o"], r["lse"], *args)
    return r, g


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("causal,window,sinks", [(True, 60, 3), (True, 33, 40), (False, 50, 4), (True, 100, 150), (False, 20, 129)])
def test_sinks_behind_the_window(kind, dim, causal, window, sinks):
    run(kind, [700], [700], 4, 2, dim, causal, window, sinks)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_sinks_of_sequences_of_different_lengths(kind):
    """the plan goes by the mean length: some sequences have nothing outside the window, one has no queries, one only the rest of a prompt"""
    run(kind, [900, 10, 0, 700, 130], [900, 10, 50, 1000, 130], 2, 1, 64, True, 40, 5)


@pytest.mark.parametrize("window,sinks", [(0, 0), (64, 2)])
def test_tiles_that_are_not_cut(window, sinks):
    """more tiles of keys than the chip has CUs: each is one block's, those with sinks are added from parts"""
    lens = [300, 1, 128, 1500] if window else [300, 129, 700, 513, 1]
    run("bf16", lens, lens, 32, 32, 64, True, window, sinks)


def test_whole_tiles_of_heads_of_128():
    run("bf16", [1300], [1300], 26, 26, 128, False, 200, 0)


def test_same_results_each_time():
    for kind in KINDS:
        (r1, g1), (r2, g2) = (run(kind, [500, 77], [500, 77], 6, 2, 64, True, 50, 3, check=False) for _ in range(2))
        assert all(torch.equal(a[n], b[n]) for a, b in ((r1, r2), (g1, g2)) for n in a)


def test_workspace_of_the_query_is_enough():
    """a workspace of exactly the size asked for, and what lies behind it, which stays"""
    heads, kv, dim, n = 4, 2, 128, 700
    q, k, v, do = rand(1, n, heads * dim, "bf16"), rand(2, n, kv * dim, "bf16"), rand(3, n, kv * dim, "bf16"), rand(4, n, heads * dim, "bf16")
    how = dict(kv_heads=kv, window=60, sinks=3)
    r = ef.attention_fwd(q, k, v, heads, **how)
    g = ef.attention_bwd(do, q, k, v, r["o"], r["lse"], heads, **how)
    need = ef.lib().efqat_attention_bwd_workspace_bytes(n, n, 1, 0, heads, kv, dim, ef.BF16, 1, 60, 3)
    pool = torch.full((need + 4096,), 77, dtype=torch.uint8, device="cuda")
    g2 = ef.attention_bwd(do, q, k, v, r["o"], r["lse"], heads, ws=pool[:need], **how)
    assert all(torch.equal(g[x], g2[x]) for x in g) and (pool[need:] == 77).all()
    with pytest.raises(ef.EfqatError):
        ef.attention_bwd(do, q, k, v, r["o"], r["lse"], heads, ws=pool[: need - 256], **how)
    lengths = torch.tensor([n], dtype=torch.int32, device="cuda")
    o = ef.attention_decode(q[:1], k[None], v[None], lengths, heads, kv_heads=kv)
    need = ef.lib().efqat_attention_decode_workspace_bytes(1, n, heads, kv, dim, 0, 0)
    pool.fill_(77)
    assert torch.equal(o, ef.attention_decode(q[:1], k[None], v[None], lengths, heads, kv_heads=kv, ws=pool[:need])) and (pool[need:] == 77).all()


def test_captured_step_and_decoding():
    """a training step and a decoding call in graphs that share no memory but their inputs, replayed with other inputs between eager calls"""
    heads, kv, dim, n = 4, 2, 64, 300
    x, do = rand(1, n, (heads + 2 * kv) * dim, "bf16"), rand(2, n, heads * dim, "bf16")
    w, pos = rand(3, 1, dim, "f32")[0], torch.arange(n, device="cuda", dtype=torch.int32)
    f = torch.rand(dim // 2, device="cuda")
    cache = [rand(s, 2 * 500, kv * dim, "bf16").view(2, 500, -1) for s in (4, 5)]
    lengths = torch.tensor([300, 41], dtype=torch.int32, device="cuda")
    cut = [heads * dim, (heads + kv) * dim]

    def train():
        q, k, v = x[:, : cut[0]], x[:, cut[0]: cut[1]], x[:, cut[1]:]
        how = dict(kv_heads=kv, q_weight=w, k_weight=w, positions=pos, inv_freq=f)
        t = ef.head_norm_rope_fwd(q, heads, k=k, **how)
        mask = dict(kv_heads=kv, window=40, sinks=2)
        r = ef.attention_fwd(t["q"], t["k"], v, heads, **mask)
        g = ef.attention_bwd(do, t["q"], t["k"], v, r["o"], r["lse"], heads, **mask)
        b = ef.head_norm_rope_bwd(g["dq"], q, heads, dk=g["dk"], k=k, **how)
        return [r["o"], r["lse"], g["dv"], *b.values()]

    def decode():
        return [ef.attention_decode(do[:2], *cache, lengths, heads, kv_heads=kv)]

    graphs = []
    for fn in (train, decode):
        fn()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = fn()
        graphs.append((fn, g, out))
    for rep in range(4):
        x.copy_(rand(10 + rep, n, x.shape[1], "bf16"))
        lengths += 7 * rep
        for fn, g, out in graphs:
            g.replay()
            eager = fn()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, eager)), (fn.__name__, rep)


def test_two_streams_at_once():
    """calls with workspaces of their own on two streams are as the calls alone"""
    heads, kv, dim, n = 8, 2, 64, 900
    sets = [[rand(10 * i + j, n, c * dim, "bf16") for j, c in enumerate((heads, kv, kv, heads))] for i in range(2)]
    how = dict(kv_heads=kv, window=100, sinks=4)

    def one(q, k, v, do):
        r = ef.attention_fwd(q, k, v, heads, **how)
        return [r["o"], *ef.attention_bwd(do, q, k, v, r["o"], r["lse"], heads, **how).values()]
    alone = [one(*s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        both = []
        for st, s in zip(streams, sets):
            with torch.cuda.stream(st):
                both.append(one(*s))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x, y in zip(alone, both) for a, b in zip(x, y))
