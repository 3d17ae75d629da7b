"""Timed cases of the operators of an attention block that lie between its quantized linear layers: norms of queries and keys for each
head with the position rotation in the same pass, attention with a sliding window and first tokens that stay visible, and dropout whose
mask is drawn from a counter and never stored.

A case is a dict of plain values:
  op        "rope"    norm (root mean square over a head) and rotation of the queries and keys of `rows` tokens
            "attn"    attention over packed sequences: forward, or forward and backward
            "decode"  attention of one new token a sequence over its cache
            "drop"    dropout of [rows][cols], forward with the residual added
  pass_     "fwd"; rope, drop: "bwd" (from what the forward took and the upstream gradient); attn: "train" (forward, then backward)
  dtype     "bf16" / "f32"
  heads, kv_heads, dim   query heads, key and value heads, features of a head
  axes      rope: positions of a token (1: text; 3: time, height, width);  freqs: rotated pairs of a head;  pairs: "half" (feature j with
            j + freqs) or "next" (2j with 2j + 1);  norm: whether heads are normed before the rotation
  seqs, rows, keys       attn: sequences, tokens of queries and of keys in all (the queries of a sequence are its last tokens); decode: `keys`
            is the room of a sequence's cache
  ragged    attn, decode: sequences of different lengths (a function of the case), else of equal ones
  causal, window, sinks  token at p sees key j: j <= p if causal; with a window, |p - j| < window or j < sinks
  cols, p   drop: columns, and the share of the elements that is dropped
"""
import math
import random
from types import SimpleNamespace

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_EPS = 1e-6
_DEFAULTS = dict(op="attn", pass_="fwd", dtype="bf16", heads=1, kv_heads=1, dim=64, axes=1, freqs=0, pairs="half", norm=True, seqs=1, rows=1,
                 keys=0, ragged=False, causal=True, window=0, sinks=0, cols=0, p=0.0)


def _case(name=None, **kw):
    c = dict(_DEFAULTS, **kw)
    if c["op"] == "attn" and not c["keys"]:
        c["keys"] = c["rows"]
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # decoding: the new tokens of a few sequences between the stacked product and the cache; a launch and a host call are what it costs
        _case("rope_fwd_decode", op="rope", rows=16, heads=32, kv_heads=8, dim=128, freqs=64),
        # a training step's backward at the LLM-sized width of 4096, weight gradients of both norms among the outputs
        _case("rope_bwd_llm", op="rope", pass_="bwd", rows=8192, heads=32, kv_heads=8, dim=128, freqs=64),
        # tokens of images and video with three positions each, neighbours paired, part of a head rotated, single precision, an odd count
        _case("rope_fwd_axes_f32", op="rope", rows=4099, heads=12, kv_heads=12, dim=80, axes=3, freqs=36, pairs="next", dtype="f32"),
        # the encoder of BERT-base: 32 sequences of 384 tokens that see each other in both directions, forward and backward
        _case("attn_train_bert", pass_="train", rows=12288, seqs=32, heads=12, kv_heads=12, dim=64, causal=False),
        # a training step of a decoder with grouped heads, window and sinks, two sequences
        _case("attn_train_window", pass_="train", rows=8192, seqs=2, heads=32, kv_heads=8, dim=128, window=1024, sinks=4),
        # fine-tuning on a few packed sequences of odd lengths in single precision
        _case("attn_train_ragged_f32", pass_="train", rows=3001, seqs=7, heads=6, kv_heads=2, dim=80, window=500, sinks=3, ragged=True, dtype="f32"),
        # evaluation of a long prompt without a window: the largest case
        _case("attn_fwd_long", rows=32768, heads=32, kv_heads=8, dim=128),
        # decoding one sequence with a long cache
        _case("decode_one", op="decode", seqs=1, keys=16384, heads=32, kv_heads=8, dim=128),
        # decoding a batch whose sequences have very different lengths
        _case("decode_batch", op="decode", seqs=64, keys=8192, heads=32, kv_heads=8, dim=128, ragged=True),
        # decoding a batch of long sequences that see a window and the first tokens; heads are not grouped
        _case("decode_window", op="decode", seqs=24, keys=6000, heads=12, kv_heads=12, dim=64, window=1024, sinks=4, ragged=True),
        # dropout of a block's output in an encoder of BERT-base, the residual added
        _case("drop_fwd_bert", op="drop", rows=12288, cols=768, p=0.1),
        # its gradient at an odd width in single precision
        _case("drop_bwd_ragged_f32", op="drop", pass_="bwd", rows=2049, cols=1001, p=0.25, dtype="f32"),
    ]


_MOST_FLOPS = 4.0 * 128 * 32 * 32768 * 32769 / 2         # the largest listed case
_MOST_VALUES = 8192 * 40 * 128                           # the largest listed tensor of an elementwise pass
_MOST_CACHE = 64 * 8192 * 8 * 128


def draw(rng):
    def size(lo, hi, steps=(1, 1, 8, 16, 64, 128)):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        step = rng.choice(steps)                         # ragged, vector-wide and tile-friendly sizes
        return min(hi, max(lo, max(1, round(v / step)) * step))

    while True:
        op = rng.choice(("rope", "rope", "attn", "attn", "attn", "decode", "decode", "drop", "drop"))
        dtype = rng.choice(("bf16", "bf16", "f32"))
        if op == "drop":
            c = _case(op=op, pass_=rng.choice(("fwd", "bwd")), rows=size(1, 32768), cols=size(8, 16384), dtype=dtype,
                      p=rng.choice((0.05, 0.1, 0.25, 0.5)))
            if c["rows"] * c["cols"] <= _MOST_VALUES:
                return c
            continue
        kv = rng.choice((1, 2, 4, 8, 12))
        heads = kv * rng.choice((1, 1, 2, 3, 4, 8))
        dim = rng.choice((64, 128, 64, 128, 32, 40, 80, 96, 112))
        if op == "rope":
            c = _case(op=op, pass_=rng.choice(("fwd", "bwd")), rows=size(1, 16384), heads=heads, kv_heads=kv, dim=dim, dtype=dtype,
                      axes=rng.choice((1, 1, 2, 3)), pairs=rng.choice(("half", "next")), norm=rng.random() < 0.8)
            c["freqs"] = rng.choice((dim // 2, dim // 2, dim // 4))
            if c["rows"] * (heads + kv) * dim <= _MOST_VALUES:
                return c
            continue
        window = rng.choice((0, size(16, 4096)))
        sinks = rng.choice((0, 1, 4, 16)) if window else 0
        if op == "decode":
            c = _case(op=op, seqs=size(1, 128, (1,)), keys=size(64, 32768), heads=heads, kv_heads=kv, dim=dim, dtype=dtype, window=window,
                      sinks=sinks, ragged=rng.random() < 0.7)
            if c["seqs"] * c["keys"] * kv * dim <= _MOST_CACHE:
                return c
            continue
        seqs = rng.choice((1, 1, 2, 5, 16))
        rows = size(1, 16384)
        if rows < 2 * seqs:
            continue
        c = _case(op=op, pass_=rng.choice(("fwd", "train", "train")), seqs=seqs, heads=heads, kv_heads=kv, dim=dim, dtype=dtype,
                  window=window, sinks=sinks, causal=rng.random() < 0.75, ragged=rng.random() < 0.6, rows=rows)
        if not c["ragged"]:
            c["rows"] = c["keys"] = rows // seqs * seqs
        if c["pass_"] == "fwd" and rng.random() < 0.3:   # the rest of a prompt whose first part is there already
            c["keys"] = c["rows"] + seqs * size(1, 4096)
        dense = 4.0 * dim * heads * sum(a * b for a, b in _lengths(c))
        if dense * (2.5 if c["pass_"] == "train" else 1.0) <= _MOST_FLOPS / 4:
            return c


def _lengths(case):
    """(queries, keys) of every sequence of an attn case; (1, keys) of a decode case."""
    c = SimpleNamespace(**{**_DEFAULTS, **case})
    rng = random.Random(c.seqs * 1000003 + c.rows * 31 + c.keys)
    if c.op == "decode":
        return [(1, rng.randint(max(1, c.keys // 16), c.keys) if c.ragged else c.keys) for _ in range(c.seqs)]
    extra = c.keys - c.rows
    if not c.ragged:
        return [(c.rows // c.seqs, c.keys // c.seqs)] * c.seqs
    cuts = sorted(rng.sample(range(1, c.rows), c.seqs - 1)) if c.seqs > 1 else []
    q = [b - a for a, b in zip([0] + cuts, cuts + [c.rows])]
    return [(n, n + extra // c.seqs) for n in q]


# ------------------------------------------------------------------ inputs
def prepare(case, seed):
    c = SimpleNamespace(**{**_DEFAULTS, **case})
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed) * 7919 + 17)
    dt = _DTYPES[c.dtype]

    def normal(*shape, std=1.0, mean=0.0):
        return torch.randn(*shape, generator=gen, device=dev, dtype=torch.float32).mul_(std).add_(mean)

    s = SimpleNamespace(c=c)
    if c.op == "drop":
        s.state = torch.randint(0, 2 ** 62, (2,), generator=gen, device=dev)
        s.x = normal(c.rows, c.cols).to(dt)
        s.residual = normal(c.rows, c.cols, std=2.0).to(dt) if c.pass_ == "fwd" else None
        return s
    nq, nk = c.heads * c.dim, c.kv_heads * c.dim
    if c.op == "rope":
        # slices of the stacked product of queries, keys and values, tokens and heads of their own width
        x = (normal(c.rows, nq + 2 * nk) * (0.5 + torch.rand(c.rows, 1, generator=gen, device=dev))).to(dt)
        s.q, s.k = x[:, :nq], x[:, nq: nq + nk]
        s.wq, s.wk = (normal(c.dim, std=0.1, mean=1.0), normal(c.dim, std=0.1, mean=1.0)) if c.norm else (None, None)
        # far positions: a batch of sequences at places of their own; the other axes are small
        far = torch.randint(0, 100000, (1, c.rows), generator=gen, device=dev, dtype=torch.int32)
        near = torch.randint(0, 64, (c.axes - 1, c.rows), generator=gen, device=dev, dtype=torch.int32)
        s.positions = torch.cat((far, near))
        s.inv_freq = (10000.0 ** (-torch.arange(c.freqs, device=dev, dtype=torch.float64) / c.freqs)).float()
        s.axis = (torch.arange(c.freqs, device=dev) * c.axes // max(c.freqs, 1)).to(torch.int32) if c.axes > 1 else None
        if c.pass_ == "bwd":
            s.dq, s.dk = normal(c.rows, nq).to(dt), normal(c.rows, nk).to(dt)
        return s
    # first keys that all queries lean towards, as trained models have them
    u = normal(c.kv_heads, 1, c.dim)
    lens = _lengths(case)

    def queries(n):
        return normal(n, c.kv_heads, c.heads // c.kv_heads, c.dim).add_(0.25 * u).view(n, nq)

    if c.op == "decode":
        s.q = queries(c.seqs).to(dt)
        k = normal(c.seqs, c.keys, c.kv_heads, c.dim).to(dt)
        k[:, :4] += u[:, 0].to(dt)
        s.k, s.v = k.view(c.seqs, c.keys, nk), normal(c.seqs, c.keys, nk).to(dt)
        s.lengths = torch.tensor([b for _, b in lens], dtype=torch.int32, device=dev)
        return s
    k = normal(c.keys, c.kv_heads, c.dim)
    at = 0
    for _, n in lens:
        k[at: at + min(4, n)] += u[:, 0]
        at += n
    k, v, q = k.view(c.keys, nk), normal(c.keys, nk), queries(c.rows)
    if c.rows == c.keys:                                 # slices of the stacked product
        x = torch.cat((q, k, v), 1).to(dt)
        s.q, s.k, s.v = x[:, :nq], x[:, nq: nq + nk], x[:, nq + nk:]
    else:
        s.q, s.k, s.v = q.to(dt), k.to(dt), v.to(dt)
    s.do = normal(c.rows, nq).to(dt) if c.pass_ == "train" else None
    s.lens = lens
    s.q_start, s.k_start = (torch.tensor([0] + [sum(l[i] for l in lens[: n + 1]) for n in range(c.seqs)], dtype=torch.int32, device=dev)
                            for i in (0, 1))
    return s


# ------------------------------------------------------------------ the passes
def run(s):
    c = s.c
    if own:
        return {"rope": _rope_own, "attn": _attn_own, "decode": _decode_own, "drop": _drop_own}[c.op](s, c)
    return {"rope": _rope_plain, "attn": _attn_plain, "decode": _decode_plain, "drop": _drop_plain}[c.op](s, c)


def _rope_own(s, c):
    import paper_2411_11038_amd as ef
    how = dict(k=s.k, kv_heads=c.kv_heads, q_weight=s.wq, k_weight=s.wk, norm=c.norm, eps=_EPS, positions=s.positions, inv_freq=s.inv_freq,
               axis=s.axis, neighbours=c.pairs == "next")
    if c.pass_ == "bwd":
        r = ef.head_norm_rope_bwd(s.dq, s.q, c.heads, dk=s.dk, **how)
        return r if c.norm else dict(dq=r["dq"], dk=r["dk"])
    return ef.head_norm_rope_fwd(s.q, c.heads, **how)


def _turn(s, c, kind):
    """Cosines and sines of the angles [rows][1][freqs]; far positions times a frequency need 64 bits."""
    pos = s.positions.to(torch.float64)
    rows = pos[s.axis.long()] if s.axis is not None else pos[:1].expand(c.freqs, -1)
    angle = rows.t() * s.inv_freq.to(torch.float64)
    return torch.cos(angle).to(kind).unsqueeze(1), torch.sin(angle).to(kind).unsqueeze(1)


def _rotate(x, cos, sin, c):
    """x [rows][heads][dim]"""
    if c.freqs == 0:
        return x
    y = x.clone()
    at = (slice(0, c.freqs), slice(c.freqs, 2 * c.freqs)) if c.pairs == "half" else (slice(0, 2 * c.freqs, 2), slice(1, 2 * c.freqs, 2))
    a, b = x[..., at[0]], x[..., at[1]]
    y[..., at[0]] = a * cos - b * sin
    y[..., at[1]] = b * cos + a * sin
    return y


def _rope_plain(s, c):
    cos, sin = _turn(s, c, torch.float32)
    out = {}
    for name, x, w, heads, dy in (("q", s.q, s.wq, c.heads, getattr(s, "dq", None)), ("k", s.k, s.wk, c.kv_heads, getattr(s, "dk", None))):
        x = x.float().view(c.rows, heads, c.dim)
        r = (x.square().mean(-1, keepdim=True) + _EPS).rsqrt() if c.norm else 1.0
        if c.pass_ == "fwd":
            out[name] = _rotate(x * r * w if c.norm else x, cos, sin, c).view(c.rows, -1).to(s.q.dtype)
            continue
        d = _rotate(dy.float().view(c.rows, heads, c.dim), cos, -sin, c)
        if c.norm:
            xhat = x * r
            g = d * w
            out["d" + name + "_weight"] = (d * xhat).sum((0, 1))
            d = r * (g - xhat * (g * xhat).mean(-1, keepdim=True))
        out["d" + name] = d.view(c.rows, -1).to(s.q.dtype)
    return out


def _attn_own(s, c):
    import paper_2411_11038_amd as ef
    how = dict(kv_heads=c.kv_heads, q_start=s.q_start, k_start=s.k_start, causal=c.causal, window=c.window, sinks=c.sinks)
    r = ef.attention_fwd(s.q, s.k, s.v, c.heads, **how)
    if c.pass_ == "train":
        r.update(ef.attention_bwd(s.do, s.q, s.k, s.v, r["o"], r["lse"], c.heads, **how))
    return r


def _seen(lo, hi, shift, keys, c, dev):
    """Which keys the queries lo .. hi - 1 of a sequence see, query i at position i + shift: bool [hi - lo][keys]."""
    p = torch.arange(lo + shift, hi + shift, device=dev).unsqueeze(1)
    j = torch.arange(keys, device=dev).unsqueeze(0)
    seen = j <= p if c.causal else torch.ones(hi - lo, keys, dtype=torch.bool, device=dev)
    if c.window:
        seen = seen & (((p - j).abs() < c.window) | (j < c.sinks))
    return seen


def _by_head(x, heads, group):
    """[n][heads * dim] -> fp32 [kv heads][group * n][dim]"""
    n = x.shape[0]
    return x.float().view(n, heads // group, group, -1).permute(1, 2, 0, 3).reshape(heads // group, group * n, -1)


def _by_token(x, n):
    """[kv heads][group * n][dim] -> [n][heads * dim]"""
    kv, m, dim = x.shape
    return x.view(kv, m // n, n, dim).permute(2, 0, 1, 3).reshape(n, -1)


def _attn_plain(s, c):
    dev, dt, group, scale = s.q.device, s.q.dtype, c.heads // c.kv_heads, c.dim ** -0.5
    train = c.pass_ == "train"
    o = torch.empty(c.rows, c.heads * c.dim, dtype=dt, device=dev)
    lse = torch.empty(c.heads, c.rows, dtype=torch.float32, device=dev)
    dq = torch.empty_like(o) if train else None
    dk, dv = (torch.empty(c.keys, c.kv_heads * c.dim, dtype=dt, device=dev) if train else None for _ in range(2))
    q0 = k0 = 0
    for nq, nk in s.lens:
        k, v = (_by_head(t[k0: k0 + nk], c.kv_heads, 1) for t in (s.k, s.v))
        kt, vt = k.transpose(1, 2).contiguous(), v.transpose(1, 2).contiguous()
        gk, gv = torch.zeros_like(k), torch.zeros_like(v)
        step = max(1, 2 ** 27 // (c.heads * nk))          # some rows of scores at a time
        for lo in range(0, nq, step):
            hi = min(nq, lo + step)
            at = slice(q0 + lo, q0 + hi)
            q = _by_head(s.q[at], c.heads, group)
            seen = _seen(lo, hi, nk - nq, nk, c, dev).repeat(group, 1)
            z = (torch.bmm(q, kt) * scale).masked_fill_(~seen, -math.inf)
            top = z.amax(-1, keepdim=True)
            e = z.sub_(top).exp_()
            total = e.sum(-1, keepdim=True)
            o[at] = _by_token(torch.bmm(e, v) / total, hi - lo).to(dt)
            lse[:, at] = (top + torch.log(total)).view(c.heads, hi - lo)
            if train:
                p = e.div_(total)
                d = _by_head(s.do[at], c.heads, group)
                dp = torch.bmm(d, vt)
                dz = p * (dp - (p * dp).sum(-1, keepdim=True)) * scale
                dq[at] = _by_token(torch.bmm(dz, k), hi - lo).to(dt)
                gk += torch.bmm(dz.transpose(1, 2).contiguous(), q)
                gv += torch.bmm(p.transpose(1, 2).contiguous(), d)
        if train:
            dk[k0: k0 + nk], dv[k0: k0 + nk] = _by_token(gk, nk).to(dt), _by_token(gv, nk).to(dt)
        q0, k0 = q0 + nq, k0 + nk
    out = dict(o=o, lse=lse)
    if train:
        out.update(dq=dq, dk=dk, dv=dv)
    return out


def _decode_own(s, c):
    import paper_2411_11038_amd as ef
    return ef.attention_decode(s.q, s.k, s.v, s.lengths, c.heads, kv_heads=c.kv_heads, window=c.window, sinks=c.sinks)


def _decode_plain(s, c):
    group = c.heads // c.kv_heads
    q = s.q.float().view(c.seqs, c.kv_heads, group, c.dim)
    j = torch.arange(c.keys, device=q.device).unsqueeze(0)
    p = s.lengths.unsqueeze(1) - 1
    seen = j <= p
    if c.window:
        seen = seen & ((p - j < c.window) | (j < c.sinks))
    o = torch.empty_like(q)
    for h in range(c.kv_heads):                          # one head of the caches at a time
        at = slice(h * c.dim, (h + 1) * c.dim)
        k, v = s.k[:, :, at].float(), s.v[:, :, at].float()
        z = torch.bmm(q[:, h], k.transpose(1, 2).contiguous()) * c.dim ** -0.5
        z = z.masked_fill(~seen.unsqueeze(1), -math.inf)
        e = torch.exp(z - z.amax(-1, keepdim=True))
        o[:, h] = torch.bmm(e, v) / e.sum(-1, keepdim=True)
    return o.view(c.seqs, -1).to(s.q.dtype)


def _drop_own(s, c):
    import paper_2411_11038_amd as ef
    if c.pass_ == "bwd":
        return ef.dropout_bwd(s.x, c.p, s.state)
    return ef.dropout_fwd(s.x, c.p, s.state, residual=s.residual)


_LOW = 0xFFFFFFFF


def _times(a, m):
    """High and low 32 bits of the product of 32-bit numbers, a in int64, m a number."""
    lo = (a & 0xFFFF) * m                                # below 2^48
    hi = (a >> 16) * m + (lo >> 16)                      # below 2^49
    return hi >> 16, ((hi & 0xFFFF) << 16) | (lo & 0xFFFF)


def _draws(state, chunks):
    """The 16-bit numbers of every chunk of 8 elements: Philox4x32 of ten rounds over (chunk, offset) with the seed as its key."""
    seed, offset = state[0], state[1]
    n = torch.arange(chunks, device=state.device)
    x = [n & _LOW, n >> 32, (offset & _LOW).expand(chunks), ((offset >> 32) & _LOW).expand(chunks)]
    k0, k1 = seed & _LOW, (seed >> 32) & _LOW
    for _ in range(10):
        h0, l0 = _times(x[0], 0xD2511F53)
        h1, l1 = _times(x[2], 0xCD9E8D57)
        x = [h1 ^ x[1] ^ k0, l1, h0 ^ x[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & _LOW, (k1 + 0xBB67AE85) & _LOW
    return torch.stack([half for w in x for half in (w & 0xFFFF, w >> 16)], 1)


def _drop_plain(s, c):
    per_row = -(-c.cols // 8)
    least = int(round(c.p * 65536))
    keep = (_draws(s.state, c.rows * per_row) >= least).view(c.rows, per_row * 8)[:, : c.cols]
    y = torch.where(keep, s.x.float() * (65536.0 / (65536 - least)), torch.zeros((), device=s.x.device))
    return (y if s.residual is None else s.residual.float() + y).to(s.x.dtype)


# ------------------------------------------------------------------ what a pass cannot do without
def _pairs(nq, nk, c):
    """(pairs of a query and a key that it sees, keys that some query sees) of a sequence and head."""
    p = torch.arange(nq, dtype=torch.int64) + (nk - nq)
    hi = torch.full_like(p, nk)
    lo = torch.zeros_like(p)
    if c.window:
        lo = (p - c.window + 1).clamp(min=0)
        hi = (p + c.window).clamp(0, nk)
    if c.causal:
        hi = torch.minimum(hi, p + 1).clamp(min=0)
    lo = torch.minimum(lo, hi)
    first = torch.minimum(lo, torch.tensor(c.sinks))
    if not c.causal and c.window:
        first = first + (min(c.sinks, nk) - hi).clamp(min=0)
    keys = int(hi.max()) - int(lo.min()) + int(first.max())
    return int((hi - lo + first).sum()), min(keys, nk)


def work(case):
    c = SimpleNamespace(**{**_DEFAULTS, **case})
    e = 2 if c.dtype == "bf16" else 4
    if c.op == "drop":
        n = float(c.rows) * c.cols
        return dict(bytes=n * e * (3 if c.pass_ == "fwd" else 2) + 16, flops=15 * n)
    if c.op == "rope":
        n = float(c.rows) * (c.heads + c.kv_heads) * c.dim
        small = 8.0 * c.dim * (2 if c.pass_ == "bwd" else 1) * c.norm + 4 * c.rows * c.axes + 4 * c.freqs
        return dict(bytes=n * e * (3 if c.pass_ == "bwd" else 2) + small, flops=(16 if c.pass_ == "bwd" else 10) * n)
    counts = [_pairs(a, b, c) for a, b in _lengths(case)]
    pairs, keys = sum(a for a, _ in counts), sum(b for _, b in counts)
    rows = c.seqs if c.op == "decode" else c.rows
    q, k = float(rows) * c.heads * c.dim * e, float(keys) * c.kv_heads * c.dim * e
    flops = 4.0 * c.dim * c.heads * pairs
    if c.op == "decode":
        return dict(bytes=2 * q + 2 * k + 4 * c.seqs, flops=flops)
    lse = 4.0 * rows * c.heads
    if c.pass_ == "fwd":
        return dict(bytes=2 * q + 2 * k + lse, flops=flops)
    # backward: scores again, then four products; q, k, v, o, do and lse in, three gradients out
    return dict(bytes=(2 * q + 2 * k + lse) + (4 * q + 4 * k + lse), flops=3.5 * flops)


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _rope_exact, "attn": _attn_exact, "decode": _decode_exact, "drop": _drop_exact}[s.c.op](s, s.c)


def _rope_exact(s, c):
    """The rotation as a product with a complex number, the backward by differentiation."""
    turn = torch.ones(c.rows, c.dim // 2, dtype=torch.complex128, device=s.q.device)
    for j in range(c.freqs):
        pos = s.positions[0 if s.axis is None else int(s.axis[j])].double()
        turn[:, j] = torch.polar(torch.ones_like(pos), pos * s.inv_freq[j].double())
    order = torch.arange(c.dim, device=s.q.device)       # pairs next to each other, features that stay behind them
    if c.pairs == "half":
        order[: 2 * c.freqs] = torch.arange(2 * c.freqs, device=s.q.device).view(2, c.freqs).t().reshape(-1)

    def forward(x, w, heads):
        x = x.view(c.rows, heads, c.dim)
        if c.norm:
            x = x / torch.sqrt(torch.linalg.vecdot(x, x)[..., None] / c.dim + _EPS) * w
        z = torch.view_as_complex(x[..., order].reshape(c.rows, heads, c.dim // 2, 2).contiguous()) * turn[:, None]
        y = torch.view_as_real(z).reshape(c.rows, heads, c.dim)
        return y[..., torch.argsort(order)].reshape(c.rows, -1)

    out = {}
    for name, x, w, heads, dy in (("q", s.q, s.wq, c.heads, getattr(s, "dq", None)), ("k", s.k, s.wk, c.kv_heads, getattr(s, "dk", None))):
        x = x.double().requires_grad_(dy is not None)
        w = w.double().requires_grad_(dy is not None) if c.norm else None
        y = forward(x, w, heads)
        if dy is None:
            out[name] = y
        elif c.norm:
            out["d" + name], out["d" + name + "_weight"] = torch.autograd.grad(y, (x, w), dy.double())
        else:
            out["d" + name], = torch.autograd.grad(y, (x,), dy.double())
    return out


def _hidden(nq, lo, hi, nk, c, dev):
    """Keys that queries lo .. hi - 1 do not see."""
    away = torch.arange(nk, device=dev)[None, :] - torch.arange(lo, hi, device=dev)[:, None] - (nk - nq)
    hidden = away > 0 if c.causal else torch.zeros_like(away, dtype=torch.bool)
    if c.window:
        outside = away.abs() >= c.window
        outside[:, : c.sinks] = False
        hidden = hidden | outside
    return hidden


def _attn_exact(s, c):
    dev, group, train = s.q.device, c.heads // c.kv_heads, c.pass_ == "train"
    o = torch.zeros(c.rows, c.heads, c.dim, dtype=torch.float64, device=dev)
    lse = torch.zeros(c.heads, c.rows, dtype=torch.float64, device=dev)
    dq = torch.zeros_like(o)
    dk, dv = (torch.zeros(c.keys, c.kv_heads, c.dim, dtype=torch.float64, device=dev) for _ in range(2))
    q0 = k0 = 0
    for nq, nk in s.lens:
        for h in range(c.heads):
            at = slice(h * c.dim, (h + 1) * c.dim)
            g = h // group
            k, v = (t[k0: k0 + nk, g * c.dim: (g + 1) * c.dim].double().requires_grad_(train) for t in (s.k, s.v))
            step = max(1, 2 ** 27 // nk)
            for lo in range(0, nq, step):
                hi = min(nq, lo + step)
                r = slice(q0 + lo, q0 + hi)
                q = s.q[r, at].double().requires_grad_(train)
                z = torch.mm(q, k.t()).div(math.sqrt(c.dim)).masked_fill(_hidden(nq, lo, hi, nk, c, dev), -math.inf)
                y = torch.mm(torch.softmax(z, 1), v)
                o[r, h], lse[h, r] = y.detach(), torch.logsumexp(z.detach(), 1)
                if train:
                    a, b, d = torch.autograd.grad(y, (q, k, v), s.do[r, at].double())
                    dq[r, h] = a
                    dk[k0: k0 + nk, g] += b
                    dv[k0: k0 + nk, g] += d
        q0, k0 = q0 + nq, k0 + nk
    out = dict(o=o.view(c.rows, -1), lse=lse)
    if train:
        out.update(dq=dq.view(c.rows, -1), dk=dk.view(c.keys, -1), dv=dv.view(c.keys, -1))
    return out


def _decode_exact(s, c):
    out = torch.zeros(c.seqs, c.heads, c.dim, dtype=torch.float64, device=s.q.device)
    group = c.heads // c.kv_heads
    for b, n in enumerate(s.lengths.tolist()):
        rows = list(range(n)) if not c.window else sorted(set(range(min(c.sinks, n))) | set(range(max(0, n - c.window), n)))
        at = torch.tensor(rows, device=s.q.device)
        k, v = (t[b, at].double().view(len(rows), c.kv_heads, c.dim).transpose(0, 1).contiguous() for t in (s.k, s.v))
        q = s.q[b].double().view(c.kv_heads, group, c.dim)
        out[b] = torch.bmm(torch.softmax(torch.bmm(q, k.transpose(1, 2).contiguous()) / math.sqrt(c.dim), -1), v).view(c.heads, c.dim)
    return out.view(c.seqs, -1)


def _drop_exact(s, c):
    """The generator in unsigned 64-bit arithmetic on the host."""
    seed, offset = (v & 0xFFFFFFFFFFFFFFFF for v in s.state.tolist())
    import numpy as np
    per_row = -(-c.cols // 8)
    low, half = np.uint64(_LOW), np.uint64(32)
    n = np.arange(c.rows * per_row, dtype=np.uint64)
    a, b = n & low, n >> half
    d, e = np.full_like(n, offset & _LOW), np.full_like(n, offset >> 32)
    k, m = seed & _LOW, seed >> 32
    for _ in range(10):
        first, second = a * np.uint64(0xD2511F53), d * np.uint64(0xCD9E8D57)
        a, b, d, e = (second >> half) ^ b ^ np.uint64(k), second & low, (first >> half) ^ e ^ np.uint64(m), first & low
        k, m = (k + 0x9E3779B9) & _LOW, (m + 0xBB67AE85) & _LOW
    words = np.stack((a, b, d, e), 1).astype("<u4")
    draws = words.view("<u2").reshape(c.rows, per_row * 8)[:, : c.cols].astype(np.int32)
    least = int(round(c.p * 65536))
    keep = torch.from_numpy(draws >= least).to(s.x.device)
    y = torch.zeros(c.rows, c.cols, dtype=torch.float64, device=s.x.device)
    y[keep] = s.x.double()[keep] / (1.0 - least / 65536.0)
    return y if s.residual is None else y + s.residual.double()
