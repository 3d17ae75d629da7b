"""The example that trains an attention block: it runs, its gradients are those of its parts in fp64, and decoding agrees with the forward."""
import numpy as np
import pytest
import torch

import paper_2411_11038_amd as ef
from oracle import attn_oracle as ao
from workloads import finetune_attention as fa

from gpu_util import host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window,sinks", [(0, 0), (24, 2)])
def test_gradients_of_a_step(window, sinks):
    heads, kv, dim = 4, 2, 64
    m, x, targets = fa.make(150, 3, heads, kv, dim, window=window, sinks=sinks, seed=2)
    weights = [host(w).copy() for w in m.qk_norm]
    r = fa.step(m, x, targets, lr=0.0)
    assert torch.isfinite(r["loss"]).all() and all(torch.isfinite(r[n].float()).all() for n in ("dx", "dboth", "datt"))
    q, k, v = (host(t).astype(np.float64) for t in fa.slices(m, r["both"]))
    t = ao.angles(m.positions.cpu().numpy()[None], host(m.inv_freq))
    tq, tk = (ao.head_norm_rope_fwd(a, n, w, True, 1e-6, t, False) for a, n, w in ((q, heads, weights[0]), (k, kv, weights[1])))
    # the attention is given queries and keys in bf16
    tq, tk = (torch.from_numpy(a).bfloat16().double().numpy() for a in (tq, tk))
    do = host(r["datt"]).astype(np.float64)
    dq, dk, dv, o = np.zeros_like(tq), np.zeros_like(tk), np.zeros_like(v), np.zeros_like(tq)
    start = m.start.cpu().numpy()
    for a, b in zip(start, start[1:]):
        mask = ao.seen(b - a, b - a, True, window, sinks)
        for h in range(heads):
            i, j = slice(h * dim, h * dim + dim), slice(h // 2 * dim, h // 2 * dim + dim)
            one, _, p = ao.attention_fwd(tq[a:b, i], tk[a:b, j], v[a:b, j], ao.default_scale(dim), mask)
            gq, gk, gv, _ = ao.attention_bwd(do[a:b, i], tq[a:b, i], tk[a:b, j], v[a:b, j], one, p, ao.default_scale(dim))
            o[a:b, i] = one
            dq[a:b, i] = gq
            dk[a:b, j] += gk
            dv[a:b, j] += gv
    gq, wq = ao.head_norm_rope_bwd(dq, q, heads, weights[0], True, 1e-6, t, False)
    gk, wk = ao.head_norm_rope_bwd(dk, k, kv, weights[1], True, 1e-6, t, False)
    # roundings to bf16, each 2^-9 of its terms in the mean: of P, dS, the gradient between the two calls and the result (independent), and the
    # queries and keys, which the two sides may round to neighbours where fp32 and fp64 fall on different sides of a tie
    got = [host(a).astype(np.float64) for a in (*fa.slices(m, r["dboth"]), r["rope"]["dq_weight"], r["rope"]["dk_weight"], r["att"])]
    for name, a, b in zip(("dq", "dk", "dv", "q weight", "k weight", "o"), got, (gq, gk, dv, wq, wk, o)):
        assert np.linalg.norm(a - b) <= 0.01 * np.linalg.norm(b), name


def test_masks_change_and_the_weights_move():
    m, x, targets = fa.make(100, 2, 2, 1, 64, drop=0.3)
    w = [m.w1.clone(), m.w2.clone(), m.head.clone(), m.qk_norm[0].clone()]
    r1, r2 = fa.step(m, x, targets, lr=0.0), fa.step(m, x, targets, lr=0.0)
    assert not torch.equal(r1["loss"], r2["loss"])               # another mask
    fa.step(m, x, targets, lr=0.1)
    assert not any(torch.equal(a, b) for a, b in zip(w, (m.w1, m.w2, m.head, m.qk_norm[0])))


def test_decoding_is_the_forward_token_by_token():
    heads, kv, dim, n, T = 4, 2, 64, 2, 40
    m, _, _ = fa.make(8, 1, heads, kv, dim, window=16, sinks=2)
    g = torch.Generator(device="cuda").manual_seed(7)
    x = torch.randn(n, T, heads * dim, generator=g, device="cuda").bfloat16()
    cache = [torch.full((n, T + 5, kv * dim), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    length = torch.zeros(n, dtype=torch.int32, device="cuda")
    out = torch.stack([fa.attend(m, x[:, t].contiguous(), cache, length) for t in range(T)], 1)
    # the cache holds the keys and values that the forward over the whole sequence would see, the queries are made again
    for s in range(n):
        q = []
        for t in range(T):                                       # as they were quantized: a range for each call
            both = fa.project(*fa.quantize(ef.layer_norm_fwd(x[:, t].contiguous(), *m.norm[0])["y"], m.w1))
            where = torch.full((n,), t, dtype=torch.int32, device="cuda")
            q.append(ef.head_norm_rope_fwd(fa.slices(m, both)[0], heads, q_weight=m.qk_norm[0], positions=where, inv_freq=m.inv_freq)["q"][s])
        ref = ef.attention_fwd(torch.stack(q), cache[0][s, :T], cache[1][s, :T], heads, kv_heads=kv, window=16, sinks=2)["o"]
        # both round P and o once: 2^-8 of |o| and of sum P |v| each
        room = 2 ** -7 * (ref.float().abs() + cache[1][s, :T].float().abs().amax())
        assert ((out[s].float() - ref.float()).abs() <= room).all()


def test_the_command_runs(capsys):
    import sys
    argv, sys.argv = sys.argv, ["finetune_attention", "--steps", "2", "--tokens", "96", "--sequences", "2"]
    try:
        fa.main()
    finally:
        sys.argv = argv
    assert "decoded 8 tokens" in capsys.readouterr().out
