"""Timed cases of the operators between the quantized linear layers of a language model: layer norm, the activation of a
feed-forward block with its inputs kept in 8 bits, and the loss over a large vocabulary, forward and backward.

A case is a dict of plain values:
  op        "norm"   layer norm of [rows][cols] over the columns, parameters in fp32
            "act"    y = f(x), or y = f(x) * up (gated), over [rows][cols]
            "xent"   softmax cross entropy of h w^T against one class a token; rows tokens of width cols, `vocab` classes
  pass_     "fwd"    forward.  norm: y and the statistics of the rows;  act: y;  xent: mean loss and log-sum-exp
            "bwd"    backward from what the forward has left
            "train"  xent only: forward, then backward
  dtype     of the activations, their gradients and the class weights ("bf16" / "f32")
  ckpt      norm, act: the forward also writes the 8-bit checkpoint of its inputs, which is then read back; a backward
            reads it in the place of the inputs (act: always)
  kind      act: "gelu" / "silu";  gated: with `up`;  packed: x and up, and their gradients, are the two halves of the rows
            of one tensor, as the product of one stacked weight leaves them
  valid     xent: share of the tokens that have a class (the others carry the ignored index)

The 8-bit checkpoint of a row: groups of 128 columns, scale = max(max|x| * fl(1/127), 2^-126) and codes rne(x * fl(1/scale)) in fp32;
codes lie in rows of whole 16 bytes.
"""
import math
from types import SimpleNamespace

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_GROUP = 128
_IGNORE = -100
_EPS = 1e-5
_DEFAULTS = dict(op="norm", pass_="fwd", rows=1, cols=1, dtype="bf16", ckpt=False, kind="gelu", gated=False, packed=False,
                 vocab=0, valid=1.0)


def _case(name=None, **kw):
    c = dict(_DEFAULTS, **kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # evaluation: one token of an LLM-sized model between two of its layers; a launch and a host call are what it costs
        _case("norm_fwd_one_token", rows=1, cols=4096),
        # the norm of a BERT-base encoder (32 sequences of 384 tokens), input kept in 8 bits and read back
        _case("norm_fwd_bert_ckpt", rows=12288, cols=768, ckpt=True),
        # its backward from the 8 bits, weight and bias gradients among the outputs
        _case("norm_bwd_bert_ckpt", pass_="bwd", rows=12288, cols=768, ckpt=True),
        # a norm of an odd width in single precision, from the kept input
        _case("norm_bwd_ragged_f32", pass_="bwd", rows=2049, cols=777, dtype="f32"),
        # evaluation: the gated activation of a few sequences decoding, one token each
        _case("act_fwd_gated_decode", op="act", rows=16, cols=11008, kind="silu", gated=True),
        # feed-forward block of the LLM-sized MLP, both inputs from one stacked product, kept in 8 bits and read back
        _case("act_fwd_gated_llm", op="act", rows=8192, cols=11008, kind="silu", gated=True, packed=True, ckpt=True),
        # its backward
        _case("act_bwd_gated_llm", op="act", pass_="bwd", rows=8192, cols=11008, kind="silu", gated=True, packed=True, ckpt=True),
        # an odd width in single precision, not gated
        _case("act_bwd_ragged_f32", op="act", pass_="bwd", rows=2049, cols=1001, dtype="f32", ckpt=True),
        # the smallest head anybody trains, single precision, a few ignored tokens
        _case("xent_train_small_f32", op="xent", pass_="train", rows=256, cols=256, vocab=1000, dtype="f32", valid=0.9),
        # masked-word training of a BERT-base encoder: one token in seven has a class, the vocabulary is no multiple of a tile
        _case("xent_train_bert_masked", op="xent", pass_="train", rows=12288, cols=768, vocab=30522, valid=0.15),
        # evaluation: the loss of a prompt of an LLM-sized model
        _case("xent_fwd_llm", op="xent", rows=2048, cols=4096, vocab=32000),
        # a training step's loss and its gradients: the largest case
        _case("xent_train_llm", op="xent", pass_="train", rows=8192, cols=4096, vocab=32000, valid=0.98),
    ]


_MOST_FLOPS = 8.0 * 8192 * 4096 * 32000    # the largest listed case
_MOST_VALUES = 8192 * 11008                # the largest listed tensor of an elementwise pass
_MOST_LOGITS = 8192 * 32000


def draw(rng):
    def size(lo, hi):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        step = rng.choice((1, 1, 8, 16, 64, 128))         # ragged, vector-wide and tile-friendly sizes
        return min(hi, max(lo, max(1, round(v / step)) * step))

    while True:
        op = rng.choice(("norm", "norm", "act", "act", "xent", "xent", "xent"))
        dtype = rng.choice(("bf16", "bf16", "f32"))
        if op == "xent":
            c = _case(op=op, pass_=rng.choice(("fwd", "train", "train")), rows=size(1, 16384), cols=size(32, 8192),
                      vocab=size(64, 131072), dtype=dtype, valid=rng.choice((1.0, 0.98, 0.9, 0.5, 0.15)))
            if 8.0 * c["rows"] * c["cols"] * c["vocab"] <= _MOST_FLOPS and c["rows"] * c["vocab"] <= _MOST_LOGITS:
                return c
            continue
        c = _case(op=op, pass_=rng.choice(("fwd", "bwd")), rows=size(1, 32768), cols=size(8, 16384), dtype=dtype)
        if c["rows"] * c["cols"] > _MOST_VALUES:
            continue
        c["ckpt"] = rng.random() < 0.5
        if op == "act":
            c["kind"] = rng.choice(("gelu", "silu"))
            c["gated"] = rng.random() < 0.6
            c["packed"] = c["gated"] and rng.random() < 0.5
            c["ckpt"] = c["ckpt"] or c["pass_"] == "bwd"
        return c


# ------------------------------------------------------------------ the 8-bit checkpoint in elementary operations
def _groups(x):
    """x [rows][cols] fp32 in groups of 128 columns, the last one filled up with zeros: [rows][groups][128]."""
    rows, cols = x.shape
    n = -(-cols // _GROUP)
    return torch.nn.functional.pad(x, (0, n * _GROUP - cols)).view(rows, n, _GROUP)


def _codes(x):
    """(codes as fp32 [rows][groups][128], scales [rows][groups])."""
    g = _groups(x.float())
    scales = (g.abs().amax(-1) * (1.0 / 127.0)).clamp_min(2.0 ** -126)
    return torch.round(g * (1.0 / scales).unsqueeze(-1)), scales


def _save(x):
    """The checkpoint as a program keeps it: int8 [rows][cols rounded up to 16], scales."""
    codes, scales = _codes(x)
    rows, cols = x.shape
    return codes.view(rows, -1)[:, : -(-cols // 16) * 16].to(torch.int8).contiguous(), scales


def _load(codes, scales, cols):
    g = _groups(codes[:, :cols].to(scales.dtype))
    return (g * scales.unsqueeze(-1)).view(codes.shape[0], -1)[:, :cols]


# ------------------------------------------------------------------ inputs
def prepare(case, seed):
    c = SimpleNamespace(**{**_DEFAULTS, **case})
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed) * 7919 + 13)
    dt = _DTYPES[c.dtype]

    def normal(*shape, std=1.0, mean=0.0):
        return torch.randn(*shape, generator=gen, device=dev, dtype=torch.float32).mul_(std).add_(mean)

    s = SimpleNamespace(c=c)
    if c.op == "xent":
        # class weights as initialised, features of unit variance that lean towards the class of their token
        w = normal(c.vocab, c.cols, std=0.02)
        target = torch.randint(0, c.vocab, (c.rows,), generator=gen, device=dev)
        sure = torch.rand(c.rows, 1, generator=gen, device=dev) * 10.0
        s.h = (normal(c.rows, c.cols) + w[target] * (sure / (c.cols * 0.0004))).to(dt)
        s.w = w.to(dt)
        ignored = torch.rand(c.rows, generator=gen, device=dev) >= c.valid
        ignored[0] = False
        s.target = torch.where(ignored, torch.full_like(target, _IGNORE), target)
        return s
    if c.op == "norm":
        # a residual stream: rows of their own offset and width
        x = (normal(c.rows, c.cols) * (0.5 + torch.rand(c.rows, 1, generator=gen, device=dev)) + normal(c.rows, 1, std=0.3)).to(dt)
        s.weight, s.bias = normal(c.cols, std=0.1, mean=1.0), normal(c.cols, std=0.1)
        if c.pass_ == "fwd":
            s.x = x
            return s
        s.dy = normal(c.rows, c.cols).to(dt)
        f = x.float()
        s.mean = f.mean(1)
        s.rstd = (f - s.mean.unsqueeze(1)).square().mean(1).add(_EPS).rsqrt()
        s.x, s.codes, s.scales = (None, *_save(x)) if c.ckpt else (x, None, None)
        return s
    both = normal(c.rows, 2 * c.cols if c.gated else c.cols, std=1.5).to(dt)
    x, up = (both[:, : c.cols], both[:, c.cols:]) if c.gated else (both, None)
    if c.pass_ == "fwd":
        s.x, s.up = (x, up) if c.packed or not c.gated else (x.contiguous(), up.contiguous())
        return s
    s.dy = normal(c.rows, c.cols).to(dt)
    s.codes, s.scales = _save(x)
    s.up_codes, s.up_scales = _save(up) if c.gated else (None, None)
    return s


# ------------------------------------------------------------------ the passes
def run(s):
    c = s.c
    if own:
        return {"norm": _norm_own, "act": _act_own, "xent": _xent_own}[c.op](s, c)
    return {"norm": _norm_plain, "act": _act_plain, "xent": _xent_plain}[c.op](s, c)


def _norm_own(s, c):
    import paper_2411_11038_amd as ef
    if c.pass_ == "bwd":
        return ef.layer_norm_bwd(s.dy, s.weight, s.mean, s.rstd, x=s.x, x_codes=s.codes, x_scales=s.scales)
    r = ef.layer_norm_fwd(s.x, s.weight, s.bias, eps=_EPS, checkpoint=c.ckpt)
    out = dict(y=r["y"], mean=r["mean"], rstd=r["rstd"])
    if c.ckpt:
        out["kept"] = ef.ckpt8_load(r["x_codes"], r["x_scales"], c.cols, s.x.dtype)
    return out


def _norm_plain(s, c):
    if c.pass_ == "bwd":
        x = _load(s.codes, s.scales, c.cols) if c.ckpt else s.x.float()
        dy = s.dy.float()
        xhat = (x - s.mean.unsqueeze(1)) * s.rstd.unsqueeze(1)
        g = dy * s.weight
        dx = (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True)) * s.rstd.unsqueeze(1)
        return dict(dx=dx.to(s.dy.dtype), dweight=(dy * xhat).sum(0), dbias=dy.sum(0))
    x = s.x.float()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = (d.square().mean(1, keepdim=True) + _EPS).rsqrt()
    out = dict(y=(d * rstd * s.weight + s.bias).to(s.x.dtype), mean=mean.squeeze(1), rstd=rstd.squeeze(1))
    if c.ckpt:
        codes, scales = _codes(x)
        out["kept"] = (codes * scales.unsqueeze(-1)).view(c.rows, -1)[:, : c.cols].to(s.x.dtype)
    return out


def _act_own(s, c):
    import paper_2411_11038_amd as ef
    kind = ef.ACT_GELU if c.kind == "gelu" else ef.ACT_SILU
    if c.pass_ == "bwd":
        if not c.packed:
            return ef.act_bwd(s.dy, kind, s.codes, s.scales, s.up_codes, s.up_scales)
        both = torch.empty(c.rows, 2 * c.cols, dtype=s.dy.dtype, device=s.dy.device)
        ef.act_bwd(s.dy, kind, s.codes, s.scales, s.up_codes, s.up_scales, out=dict(dx=both[:, : c.cols], dup=both[:, c.cols:]))
        return both
    r = ef.act_fwd(s.x, kind, up=s.up, checkpoint=c.ckpt)
    out = dict(y=r["y"])
    if c.ckpt:
        out["kept"] = ef.ckpt8_load(r["x_codes"], r["x_scales"], c.cols, s.x.dtype)
        if c.gated:
            out["up_kept"] = ef.ckpt8_load(r["up_codes"], r["up_scales"], c.cols, s.x.dtype)
    return out


def _act_plain(s, c):
    def value_and_slope(x):
        if c.kind == "gelu":
            half = 0.5 * (1.0 + torch.erf(x * math.sqrt(0.5)))
            return x * half, half + x * torch.exp(-0.5 * x * x) * math.sqrt(0.5 / math.pi)
        sig = 1.0 / (1.0 + torch.exp(-x))
        return x * sig, sig * (1.0 + x * (1.0 - sig))

    if c.pass_ == "bwd":
        f, slope = value_and_slope(_load(s.codes, s.scales, c.cols))
        dy, dt = s.dy.float(), s.dy.dtype
        if not c.gated:
            return dict(dx=(dy * slope).to(dt), dup=None)
        dx, dup = dy * slope * _load(s.up_codes, s.up_scales, c.cols), dy * f
        return torch.cat((dx, dup), 1).to(dt) if c.packed else dict(dx=dx.to(dt), dup=dup.to(dt))
    x = s.x.float()
    if c.kind == "gelu":
        y = x * (0.5 * (1.0 + torch.erf(x * math.sqrt(0.5))))
    else:
        y = x / (1.0 + torch.exp(-x))
    if c.gated:
        y = y * s.up.float()
    out = dict(y=y.to(s.x.dtype))
    if c.ckpt:
        for name, t in (("kept", s.x), ("up_kept", s.up if c.gated else None)):
            if t is not None:
                codes, scales = _codes(t)
                out[name] = (codes * scales.unsqueeze(-1)).view(c.rows, -1)[:, : c.cols].to(t.dtype)
    return out


def _xent_own(s, c):
    import paper_2411_11038_amd as ef
    r = ef.linear_xent_fwd(s.h, s.w, s.target, ignore_index=_IGNORE)
    if c.pass_ == "train":
        r.update(ef.linear_xent_bwd(s.h, s.w, s.target, r["lse"], ignore_index=_IGNORE))
    return r


def _xent_plain(s, c):
    h, w = s.h.float(), s.w.float()
    valid = s.target != _IGNORE
    t = torch.where(valid, s.target, torch.zeros_like(s.target)).unsqueeze(1)
    n = valid.sum()
    z = h @ w.t()
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    lse = top + torch.log(total)
    loss = torch.where(valid, (lse - z.gather(1, t)).squeeze(1), torch.zeros_like(lse[:, 0])).sum() / n
    out = dict(loss=loss.view(1), lse=torch.where(valid, lse.squeeze(1), torch.zeros_like(lse[:, 0])),
               n_valid=n.to(torch.int32).view(1))
    if c.pass_ == "train":
        g = e.div_(total)
        g.scatter_add_(1, t, torch.full_like(total, -1.0))
        g.mul_((valid.to(torch.float32) / n).unsqueeze(1))
        out.update(dh=(g @ w).to(s.h.dtype), dw=(g.t() @ h).to(s.w.dtype))
    return out


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = SimpleNamespace(**{**_DEFAULTS, **case})
    e = 2 if c.dtype == "bf16" else 4
    n = float(c.rows) * c.cols
    kept = c.rows * (-(-c.cols // 16) * 16 + 4.0 * -(-c.cols // _GROUP))      # codes and scales of one tensor
    if c.op == "norm":
        if c.pass_ == "fwd":
            return dict(bytes=2 * n * e + 8 * c.cols + 8 * c.rows + (2 * kept + n * e if c.ckpt else 0), flops=8 * n)
        return dict(bytes=2 * n * e + (kept if c.ckpt else n * e) + 12 * c.cols + 8 * c.rows, flops=14 * n)
    if c.op == "act":
        m = 2 if c.gated else 1
        if c.pass_ == "fwd":
            return dict(bytes=(m + 1) * n * e + (m * (2 * kept + n * e) if c.ckpt else 0), flops=20 * n)
        return dict(bytes=(m + 1) * n * e + m * kept, flops=30 * n)
    # logits of the tokens that have a class; the backward forms them again, as they are not kept, and multiplies twice more
    t = max(1.0, c.rows * c.valid)
    weights, features = float(c.vocab) * c.cols * e, t * c.cols * e
    fwd = dict(bytes=weights + features + 8 * c.rows + 4 * t, flops=2 * t * c.cols * c.vocab)
    if c.pass_ == "fwd":
        return fwd
    return dict(bytes=fwd["bytes"] + 2 * weights + features + c.rows * c.cols * e + 12 * c.rows, flops=4 * fwd["flops"])


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _norm_exact, "act": _act_exact, "xent": _xent_exact}[s.c.op](s, s.c)


def _kept_exact(x):
    """What the codes stand for: the codes are defined by their fp32 rounding, the rest is exact."""
    rows, cols = x.shape
    out = torch.empty(rows, cols, dtype=torch.float64, device=x.device)
    for lo in range(0, cols, _GROUP):
        part = x[:, lo: lo + _GROUP].to(torch.float32)
        scale = torch.maximum(part.abs().max(dim=1, keepdim=True).values * (1.0 / 127.0), torch.tensor(2.0 ** -126, device=x.device))
        out[:, lo: lo + _GROUP] = torch.round(part * torch.reciprocal(scale)).double() * scale.double()
    return out


def _norm_exact(s, c):
    w = s.weight.double()
    if c.pass_ == "fwd":
        x = s.x.double()
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = 1.0 / torch.sqrt(var + _EPS)
        out = dict(y=(x - mean[:, None]) * rstd[:, None] * w + s.bias.double(), mean=mean, rstd=rstd)
        if c.ckpt:
            out["kept"] = _kept_exact(s.x)
        return out
    x = s.codes[:, : c.cols].double() * s.scales.double().repeat_interleave(_GROUP, 1)[:, : c.cols] if c.ckpt else s.x.double()
    dy, rstd = s.dy.double(), s.rstd.double()
    xhat = (x - s.mean.double()[:, None]) * rstd[:, None]
    g = dy * w
    sum_g, sum_gx = g.sum(1), torch.linalg.vecdot(g, xhat)
    dx = rstd[:, None] / c.cols * (c.cols * g - sum_g[:, None] - xhat * sum_gx[:, None])
    return dict(dx=dx, dweight=torch.linalg.vecdot(dy, xhat, dim=0), dbias=dy.sum(0))


def _act_exact(s, c):
    def cdf(x):
        return torch.special.ndtr(x) if c.kind == "gelu" else torch.sigmoid(x)

    if c.pass_ == "fwd":
        y = s.x.double() * cdf(s.x.double())
        out = dict(y=y * s.up.double() if c.gated else y)
        if c.ckpt:
            out["kept"] = _kept_exact(s.x)
            if c.gated:
                out["up_kept"] = _kept_exact(s.up)
        return out
    x = s.codes[:, : c.cols].double() * s.scales.double().repeat_interleave(_GROUP, 1)[:, : c.cols]
    p, dy = cdf(x), s.dy.double()
    slope = p + (x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi) if c.kind == "gelu" else x * p * (1 - p))
    if not c.gated:
        return dict(dx=dy * slope, dup=None)
    up = s.up_codes[:, : c.cols].double() * s.up_scales.double().repeat_interleave(_GROUP, 1)[:, : c.cols]
    dx, dup = dy * slope * up, dy * x * p
    return torch.cat((dx, dup), 1) if c.packed else dict(dx=dx, dup=dup)


def _xent_exact(s, c):
    rows = torch.nonzero(s.target != _IGNORE).squeeze(1)
    n = rows.numel()
    w = s.w.double()
    lse = torch.zeros(c.rows, dtype=torch.float64, device=w.device)
    loss = torch.zeros((), dtype=torch.float64, device=w.device)
    train = c.pass_ == "train"
    dh = torch.zeros(c.rows, c.cols, dtype=torch.float64, device=w.device) if train else None
    dw = torch.zeros_like(w) if train else None
    for lo in range(0, n, 1024):                      # some tokens at a time
        r = rows[lo: lo + 1024]
        h, t = s.h[r].double(), s.target[r]
        z = torch.mm(h, w.t().contiguous())
        lse[r] = torch.logsumexp(z, 1)
        loss += (lse[r] - z[torch.arange(r.numel(), device=z.device), t]).sum()
        if train:
            g = torch.exp(z - lse[r][:, None])
            g[torch.arange(r.numel(), device=z.device), t] -= 1.0
            g /= n
            dh[r] = torch.mm(g, w)
            dw += torch.mm(g.t().contiguous(), h)
    out = dict(loss=(loss / n).view(1), lse=lse, n_valid=None)
    if train:
        out.update(dh=dh, dw=dw)
    return out
