#!/usr/bin/env python3
"""One attention block of a language model, its head and its loss, trained with the calls of this library alone: norms of queries and keys with the
position rotation, attention with a window and first tokens that stay visible, and dropout next to the restricted backward of the
quantized linear layers; and the same block decoding token by token over its cache.

    python -m workloads.finetune_attention [--tokens 512 --sequences 4 --heads 4 --kv-heads 2 --dim 64 --window 64 --sinks 2 --steps 30]

    x -> layer norm -> codes -> W1 (queries, keys and values, one stacked weight) -> norms, rotation -> attention -> codes -> W2 -> dropout, + x
      -> layer norm -> head, loss

Of W1 and W2 the most important fraction of the rows is updated (by the step that is fused into their backward call), of the norms and the
head everything.  Synthetic data: every token's class is a fixed function of its features and of those of the token before it."""
from __future__ import annotations

import argparse
from types import SimpleNamespace

import torch

import paper_2411_11038_amd as ef


def make(tokens, sequences, heads, kv_heads, dim, vocab=200, window=0, sinks=0, drop=0.1, seed=0, device="cuda"):
    g = torch.Generator(device=device).manual_seed(seed)
    rand = lambda *s, std=1.0: torch.randn(*s, generator=g, device=device) * std
    m = SimpleNamespace(heads=heads, kv_heads=kv_heads, dim=dim, window=window, sinks=sinks, drop=drop)
    width = heads * dim
    m.w1, m.w2 = rand((heads + 2 * kv_heads) * dim, width, std=width ** -0.5), rand(width, width, std=width ** -0.5)
    m.head = rand(vocab, width, std=0.02)                        # fp32 master weights; the products take a bf16 copy
    m.norm = [[torch.ones(width, device=device), torch.zeros(width, device=device)] for _ in range(2)]
    m.qk_norm = [torch.ones(dim, device=device) for _ in range(2)]
    m.inv_freq = (10000.0 ** (-torch.arange(dim // 2, device=device) / (dim // 2))).float()
    m.adam = [dict(adam_m=torch.zeros(w.shape[0], device=device), adam_v=torch.zeros(w.shape[0], device=device),
                   adam_t=torch.zeros(w.shape[0], dtype=torch.int32, device=device)) for w in (m.w1, m.w2)]
    m.state = torch.tensor([seed, 0], dtype=torch.int64, device=device)      # dropout: seed, and the steps as offset
    x = rand(tokens, width).bfloat16()
    # sequences of different lengths, packed
    cuts = torch.linspace(0, 1, sequences + 1) ** 1.3 * tokens
    m.start = cuts.round().to(torch.int32).to(device)
    m.positions = torch.arange(tokens, device=device, dtype=torch.int32)
    m.positions -= m.start[torch.searchsorted(m.start[1:].contiguous(), m.positions, right=True)]
    targets = ((x + x.roll(1, 0)).float() @ rand(width, vocab)).argmax(1)
    return m, x, targets


def slices(m, both):
    """queries, keys, values of the stacked product"""
    a, b = m.heads * m.dim, (m.heads + m.kv_heads) * m.dim
    return both[:, :a], both[:, a:b], both[:, b:]


def rope(m, positions):
    return dict(kv_heads=m.kv_heads, q_weight=m.qk_norm[0], k_weight=m.qk_norm[1], positions=positions, inv_freq=m.inv_freq)


def quantize(a, w, num=1, den=4, bits=8):
    return ef.fakequant_fwd(a, ef.ACT_PER_TENSOR_ASYM, 8), ef.weight_quant_select(w, bits, ef.k_from_ratio(w.shape[0], num, den))


def project(qa, qw):
    return ef.linear_fwd(qa["codes"], qa["scale"], qa["zero_point"], qw["codes"], qw["scale"])


def step(m, x, targets, num=1, den=4, lr=0.2, lr_scale=1e-4):
    """One training step; returns the loss and the gradients that are not applied by the fused step, with what they were made from."""
    mask = dict(kv_heads=m.kv_heads, q_start=m.start, window=m.window, sinks=m.sinks)
    m.state[1] += 1                                              # another mask

    def backward(dy, a, qa, w, qw, adam):
        r = ef.linear_bwd(dy, qa["codes"], qa["clip_bits"], a, qa["scale"], qa["zero_point"], qw["codes"], qw["clip_bits"], w,
                          qw["scale"], qw["idx"], step=dict(lr_w=lr, lr_s=lr_scale, **adam))
        return r["dx"]

    # forward
    n1 = ef.layer_norm_fwd(x, *m.norm[0], checkpoint=True)
    q1, k1 = quantize(n1["y"], m.w1, num, den)
    both = project(q1, k1)
    q, k, v = slices(m, both)
    turned = ef.head_norm_rope_fwd(q, m.heads, k=k, **rope(m, m.positions))
    att = ef.attention_fwd(turned["q"], turned["k"], v, m.heads, **mask)
    q2, k2 = quantize(att["o"], m.w2, num, den)
    h = ef.dropout_fwd(project(q2, k2), m.drop, m.state, residual=x)
    n2 = ef.layer_norm_fwd(h, *m.norm[1], checkpoint=True)
    head = m.head.bfloat16()
    loss = ef.linear_xent_fwd(n2["y"], head, targets)

    # backward
    d = ef.linear_xent_bwd(n2["y"], head, targets, loss["lse"])
    g2 = ef.layer_norm_bwd(d["dh"], m.norm[1][0], n2["mean"], n2["rstd"], x_codes=n2["x_codes"], x_scales=n2["x_scales"])
    datt = backward(ef.dropout_bwd(g2["dx"], m.drop, m.state), att["o"], q2, m.w2, k2, m.adam[1])
    dboth = torch.empty_like(both)
    dq, dk, dv = slices(m, dboth)
    ga = ef.attention_bwd(datt, turned["q"], turned["k"], v, att["o"], att["lse"], m.heads, **mask, out=dict(dq=dq, dk=dk, dv=dv))
    gr = ef.head_norm_rope_bwd(dq, q, m.heads, dk=dk, k=k, **rope(m, m.positions), out=dict(dq=dq, dk=dk))
    dn1 = backward(dboth, n1["y"], q1, m.w1, k1, m.adam[0])
    g1 = ef.layer_norm_bwd(dn1, m.norm[0][0], n1["mean"], n1["rstd"], x_codes=n1["x_codes"], x_scales=n1["x_scales"])
    dx = g1["dx"] + g2["dx"]

    # norms and head are never frozen
    m.head.sub_(d["dw"], alpha=lr)
    for p, g in zip(m.norm, (g1, g2)):
        p[0].sub_(g["dweight"], alpha=lr)
        p[1].sub_(g["dbias"], alpha=lr)
    for p, g in zip(m.qk_norm, (gr["dq_weight"], gr["dk_weight"])):
        p.sub_(g, alpha=lr)
    return dict(loss=loss["loss"], dx=dx, both=both, dboth=dboth, datt=datt, att=att["o"], rope=gr, dres=g2["dx"])


def attend(m, x, cache, length):
    """The block's attention for one new token a sequence, x [sequences, width]: its keys and values go to place length[s] of the cache
    (k, v: [sequences, capacity, kv_heads * dim]).  length: int32 [sequences], advanced."""
    both = project(*quantize(ef.layer_norm_fwd(x, *m.norm[0])["y"], m.w1))
    q, k, v = slices(m, both)
    ef.head_norm_rope_fwd(q, m.heads, k=k, **rope(m, length), out=dict(q=q, k=k))         # where they lie
    at = length.long()
    rows = torch.arange(x.shape[0], device=x.device)
    cache[0][rows, at], cache[1][rows, at] = k, v
    length += 1
    return ef.attention_decode(q, cache[0], cache[1], length, m.heads, kv_heads=m.kv_heads, window=m.window, sinks=m.sinks)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("tokens", 512), ("sequences", 4), ("heads", 4), ("kv-heads", 2), ("dim", 64), ("window", 64), ("sinks", 2), ("steps", 30)):
        ap.add_argument("--" + name, type=int, default=default)
    a = ap.parse_args()
    m, x, targets = make(a.tokens, a.sequences, a.heads, a.kv_heads, a.dim, window=a.window, sinks=a.sinks)
    for i in range(a.steps):
        r = step(m, x, targets)
        if i % 5 == 0 or i == a.steps - 1:
            print(f"step {i:3d}  loss {float(r['loss']):.4f}", flush=True)
    capacity, n = 32, 3
    cache = [torch.zeros(n, capacity, a.kv_heads * a.dim, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    length = torch.zeros(n, dtype=torch.int32, device="cuda")
    for i in range(8):
        o = attend(m, x[i * n: (i + 1) * n], cache, length)
    print(f"decoded {i + 1} tokens of {n} sequences, output {tuple(o.shape)}")


if __name__ == "__main__":
    main()
