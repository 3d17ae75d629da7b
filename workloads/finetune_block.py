#!/usr/bin/env python3
"""One feed-forward block of a language model, its head and its loss, trained with the calls of this library alone: what lies between the
quantized linear layers (layer norm, gated activation, cross entropy) next to the restricted backward of those layers.

    python -m workloads.finetune_block [--tokens 512 --width 256 --hidden 688 --vocab 1000 --steps 30 --fraction 1/4]

    x -> layer norm -> codes -> W1 (gate and up, one stacked weight) -> SiLU(gate) * up -> codes -> W2 -> + x -> layer norm -> head, loss

Forward, the layer norms and the activation keep their inputs in 8 bits; backward reads those.  Of W1 and W2 the most important
fraction of the rows is updated (by the step that is fused into their backward call), of the norms and the head everything.  Synthetic
data: every token's class is a fixed function of its features."""
from __future__ import annotations

import argparse
from types import SimpleNamespace

import torch

import paper_2411_11038_amd as ef


def make(tokens, width, hidden, vocab, ignored=0.1, seed=0, device="cuda"):
    g = torch.Generator(device=device).manual_seed(seed)
    rand = lambda *s, std=1.0: torch.randn(*s, generator=g, device=device) * std
    m = SimpleNamespace()
    m.w1, m.w2 = rand(2 * hidden, width, std=width ** -0.5), rand(width, hidden, std=hidden ** -0.5)
    m.head = rand(vocab, width, std=0.02)                        # fp32 master weights; the products take a bf16 copy
    m.norm = [[torch.ones(width, device=device), torch.zeros(width, device=device)] for _ in range(2)]
    m.adam = [dict(adam_m=torch.zeros(w.shape[0], device=device), adam_v=torch.zeros(w.shape[0], device=device),
                   adam_t=torch.zeros(w.shape[0], dtype=torch.int32, device=device)) for w in (m.w1, m.w2)]
    x = rand(tokens, width).bfloat16()
    targets = (x.float() @ rand(width, vocab)).argmax(1)
    targets[torch.rand(tokens, generator=g, device=device) < ignored] = -100
    return m, x, targets


def step(m, x, targets, num=1, den=4, lr=0.2, lr_scale=1e-4, bits=8):
    """One training step; returns dict(loss, n_valid) and the gradients that are not applied by the fused step."""
    hidden, width = m.w2.shape[1], m.w2.shape[0]

    def quantize(a, w):
        qa = ef.fakequant_fwd(a, ef.ACT_PER_TENSOR_ASYM, 8)
        k = ef.k_from_ratio(w.shape[0], num, den)
        return qa, ef.weight_quant_select(w, bits, k)

    def backward(dy, a, qa, w, qw, adam):
        r = ef.linear_bwd(dy, qa["codes"], qa["clip_bits"], a, qa["scale"], qa["zero_point"], qw["codes"], qw["clip_bits"], w,
                          qw["scale"], qw["idx"], step=dict(lr_w=lr, lr_s=lr_scale, **adam))
        return r["dx"]

    # forward
    n1 = ef.layer_norm_fwd(x, *m.norm[0], checkpoint=True)
    q1, k1 = quantize(n1["y"], m.w1)
    both = ef.linear_fwd(q1["codes"], q1["scale"], q1["zero_point"], k1["codes"], k1["scale"])
    act = ef.act_fwd(both[:, :hidden], ef.ACT_SILU, up=both[:, hidden:], checkpoint=True)
    del both                                                     # 8 bits of it are kept
    q2, k2 = quantize(act["y"], m.w2)
    h = x + ef.linear_fwd(q2["codes"], q2["scale"], q2["zero_point"], k2["codes"], k2["scale"])
    n2 = ef.layer_norm_fwd(h, *m.norm[1], checkpoint=True)
    head = m.head.bfloat16()
    loss = ef.linear_xent_fwd(n2["y"], head, targets)

    # backward
    d = ef.linear_xent_bwd(n2["y"], head, targets, loss["lse"])
    g2 = ef.layer_norm_bwd(d["dh"], m.norm[1][0], n2["mean"], n2["rstd"], x_codes=n2["x_codes"], x_scales=n2["x_scales"])
    dact = backward(g2["dx"], act["y"], q2, m.w2, k2, m.adam[1])
    dboth = torch.empty(x.shape[0], 2 * hidden, dtype=x.dtype, device=x.device)
    ef.act_bwd(dact, ef.ACT_SILU, act["x_codes"], act["x_scales"], act["up_codes"], act["up_scales"],
               out=dict(dx=dboth[:, :hidden], dup=dboth[:, hidden:]))
    dn1 = backward(dboth, n1["y"], q1, m.w1, k1, m.adam[0])
    g1 = ef.layer_norm_bwd(dn1, m.norm[0][0], n1["mean"], n1["rstd"], x_codes=n1["x_codes"], x_scales=n1["x_scales"])
    dx = g1["dx"] + g2["dx"]

    # norms and head are never frozen
    m.head.sub_(d["dw"], alpha=lr)
    for p, g in zip(m.norm, (g1, g2)):
        p[0].sub_(g["dweight"], alpha=lr)
        p[1].sub_(g["dbias"], alpha=lr)
    return dict(loss=loss["loss"], n_valid=loss["n_valid"], dx=dx, dhead=d["dw"], norms=(g1, g2))


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("tokens", 512), ("width", 256), ("hidden", 688), ("vocab", 1000), ("steps", 30)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--fraction", default="1/4", help="rows of the linear layers that are updated")
    a = ap.parse_args()
    num, den = (int(v) for v in a.fraction.split("/"))
    m, x, targets = make(a.tokens, a.width, a.hidden, a.vocab)
    for i in range(a.steps):
        r = step(m, x, targets, num, den)
        if i % 5 == 0 or i == a.steps - 1:
            print(f"step {i:3d}  loss {float(r['loss']):.4f}  ({int(r['n_valid'])} tokens with a class)", flush=True)


if __name__ == "__main__":
    main()
