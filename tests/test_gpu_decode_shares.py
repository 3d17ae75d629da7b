"""Decoding whose keys are cut into several shares: as many as 64, some of them empty, cut beside the gap between first tokens and window; heads of 80 and
96 features in one share and in several."""
import numpy as np
import pytest
import torch

import paper_2411_11038_amd as ef
from oracle import attn_oracle as ao

import attn_checks as ck
from gpu_util import host

pytestmark = pytest.mark.gpu
KINDS = {"bf16": torch.bfloat16, "f32": torch.float32}


def rand(seed, rows, cols, kind, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(rows, cols, generator=g, device="cuda") * std).to(KINDS[kind])


def shares_of(n, cap, heads, kv, dim, window, sinks):
    """what the workspace has room for: a row of 64 or 128 features and 4 more for each head and share"""
    need = ef.lib().efqat_attention_decode_workspace_bytes(n, cap, heads, kv, dim, window, sinks)
    each = n * heads * ((64 if dim <= 64 else 128) + 4) * 4
    return max(1, need // each)


#        capacity, lengths, heads, kv heads, dim, window, sinks, shares
CASES = [(1500, [1500, 1, 0, 33, 700], 4, 2, 64, 0, 0, 3),
         (2000, [1999, 64, 2000], 6, 3, 128, 0, 0, 4),
         (2500, [2500, 31, 1200], 8, 2, 96, 0, 0, 5),
         (2500, [2100, 2500], 40, 1, 80, 0, 0, 5),
         (16384, [16384, 500], 4, 2, 128, 0, 0, 32),
         (32768, [32768, 40, 20000], 2, 1, 96, 0, 0, 64),
         (32768, [31111], 1, 1, 64, 0, 0, 64),
         (6000, [6000, 3100, 20, 5000], 4, 2, 128, 3000, 40, 7),
         (6000, [5990, 70, 0], 3, 1, 40, 2000, 1, 5),
         (6000, [5990, 700], 2, 2, 96, 1000, 300, 3),
         (400, [400, 1, 0, 399], 4, 2, 80, 0, 0, 1),
         (400, [400, 33, 31], 3, 3, 96, 0, 0, 1),
         (400, [400, 300, 32], 5, 1, 96, 50, 3, 1),
         (1000, [1000, 517], 4, 4, 112, 0, 0, 2)]


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_shares(kind, case):
    cap, lens, heads, kv, dim, window, sinks, shares = CASES[case]
    n = len(lens)
    got = shares_of(n, cap, heads, kv, dim, window, sinks)
    assert got == shares, f"{got} shares"
    q = rand(1, n, heads * dim, kind, 1.5)
    k, v = (rand(s, n * cap, kv * dim, kind).view(n, cap, -1) for s in (2, 3))
    for s, m in enumerate(lens):
        k[s, m:] = float("nan")                              # a cache holds anything there
        v[s, m:] = float("inf")
    # a workspace that held something else
    ws = torch.full((ef.lib().efqat_attention_decode_workspace_bytes(n, cap, heads, kv, dim, window, sinks),), 255, dtype=torch.uint8, device="cuda")
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    o = ef.attention_decode(q, k, v, lengths, heads, kv_heads=kv, window=window, sinks=sinks, ws=ws)
    scale, u, E = ao.default_scale(dim), ck.half_step(kind), ck.E
    for s, m in enumerate(lens):
        if m == 0:
            assert (o[s] == 0).all()
            continue
        O, Q, K, V = ck.heads_of(o[s: s + 1], heads), ck.heads_of(q[s: s + 1], heads), ck.heads_of(k[s, :m], kv), ck.heads_of(v[s, :m], kv)
        mask = ao.seen(1, m, True, window, sinks)
        for h in range(heads):
            g = h * kv // heads
            ref, lse, p = ao.attention_fwd(Q[h], K[g], V[g], scale, mask)
            size = scale * (np.abs(Q[h]) @ np.abs(K[g]).T)
            eta = np.where(mask, ck._spread(size, lse, dim), 0.0)
            # sums of m terms and of the shares; each term has the factors of its wavefront, its block and its share, four half steps and the
            # argument's error (in eta) each
            fine = p * (eta + 3 * eta.max() + (m + shares + 8 + 32) * E)
            ck.within(O[h], ref, 1.01 * u * np.abs(ref) + 1.01 * (p * u + fine) @ np.abs(V[g]) + 1e-30, f"sequence {s} head {h}")
            if kind == "bf16":
                ck.near(O[h], ref, u * np.sqrt(ref ** 2 + p ** 2 @ V[g] ** 2), fine @ np.abs(V[g]), f"sequence {s} head {h}")


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_every_share_has_its_weight(kind):
    """16384 keys in 32 shares, all scores zero: values that say which 256 keys they belong to"""
    cap, dim = 16384, 64
    assert shares_of(1, cap, 2, 1, dim, 0, 0) == 32
    q, k = torch.zeros(1, 2 * dim, device="cuda", dtype=KINDS[kind]), torch.zeros(1, cap, dim, device="cuda", dtype=KINDS[kind])
    v = torch.zeros(1, cap, dim, device="cuda", dtype=KINDS[kind])
    at = torch.arange(cap, device="cuda")
    v[0, at, at // 256] = 1
    for m in (16384, 16383, 8191, 300, 1):
        o = host(ef.attention_decode(q, k, v, torch.tensor([m], dtype=torch.int32, device="cuda"), 2, kv_heads=1))
        count = np.clip(m - 256 * np.arange(dim), 0, 256) / m        # whole numbers until the quotient: rounded once or twice
        assert (np.abs(o.reshape(2, dim) - count) <= (ck.half_step(kind) + 2 * ck.E) * count).all(), m


def test_replayed_with_other_lengths():
    """a captured call over 32 shares: sequences grow and shrink between replays, shares fill and empty"""
    n, cap, heads, kv, dim = 2, 16384, 4, 2, 128
    q, k, v = rand(1, n, heads * dim, "bf16"), rand(2, n * cap, kv * dim, "bf16").view(n, cap, -1), rand(3, n * cap, kv * dim, "bf16").view(n, cap, -1)
    assert shares_of(n, cap, heads, kv, dim, 0, 0) == 32
    lengths = torch.tensor([16384, 10], dtype=torch.int32, device="cuda")
    ef.attention_decode(q, k, v, lengths, heads, kv_heads=kv)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = ef.attention_decode(q, k, v, lengths, heads, kv_heads=kv)
    for lens in ((16384, 10), (0, 16384), (5, 5), (9000, 1), (16384, 16383)):
        lengths.copy_(torch.tensor(lens, dtype=torch.int32))
        graph.replay()
        eager = ef.attention_decode(q, k, v, lengths, heads, kv_heads=kv)
        torch.cuda.synchronize()
        assert torch.equal(o, eager), lens
