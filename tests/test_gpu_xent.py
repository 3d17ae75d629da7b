"""Softmax cross entropy over a vocabulary against the fp64 definition.

Bounds, element by element, from what the arithmetic may lose (e = 2^-24; sums of n terms in fp32 over registers, lanes and tiles lose
far less than sqrt(n) e of the sum of magnitudes each; 2e-6 = 32 e is taken):
  z      dz = 2e-6 max_tv sum_k |h_k w_k|
  lse, loss   dz + 4e-6 (1 + |lse|)
  G      relative to p: dz + 4e-6 (1 + |lse|); bf16 operands: 2^-8 of |G| more, its rounding
  dh     sum_v dG |w| + 4e-6 sum_v |G w|, dw alike; bf16 results: 2^-8 of the value more"""
import numpy as np
import pytest
import torch

import paper_2411_11038_amd as ef
from oracle import lm_oracle as lo

from gpu_util import act_tensor, host, report

pytestmark = pytest.mark.gpu


def make(T, D, V, dtype, seed, ignored=0.0, std=None):
    rng = np.random.default_rng(seed)
    w = rng.standard_normal((V, D)).astype(np.float32) * np.float32(std or 2.0 / np.sqrt(D))
    t = rng.integers(0, V, T)
    h = (rng.standard_normal((T, D)) + 0.6 * rng.random((T, 1)) * np.sqrt(D) * w[t]).astype(np.float32)
    t = np.where(rng.random(T) < ignored, -100, t)
    hd, wd = act_tensor(h, dtype), act_tensor(w, dtype)
    return host(hd).astype(np.float32), host(wd).astype(np.float32), t, hd, wd, torch.from_numpy(t).cuda()


def check_all(h, w, t, hd, wd, td, dtype, reduction=ef.XENT_MEAN, dloss=None, ignore=-100, **kw):
    T, V = len(t), w.shape[0]
    has = (t != ignore) & (t >= 0) & (t < V)
    n = int(has.sum())
    r = ef.linear_xent_fwd(hd, wd, td, ignore_index=ignore, reduction=reduction)
    up = torch.from_numpy(dloss.astype(np.float32)).cuda() if dloss is not None else None
    r.update(ef.linear_xent_bwd(hd, wd, td, r["lse"], dloss=up, ignore_index=ignore, reduction=reduction, **kw))
    scale = np.ones(T) if dloss is None else np.broadcast_to(dloss.astype(np.float32).astype(np.float64), (T,))
    if reduction == ef.XENT_MEAN:
        scale = scale / max(n, 1)
    loss, lse, p, g = lo.xent(np.where(has[:, None], h, 0.0), w, t, ignore, scale)
    a, b = np.abs(np.where(has[:, None], h, 0.0)).astype(np.float64), np.abs(w).astype(np.float64)
    dz = 2e-6 * (a @ b.T).max() if n else 0.0
    d_lse = dz + 4e-6 * (1 + np.abs(lse))
    assert int(r["n_valid"]) == n
    ratio = {}

    def within(name, got, ref, bound):
        err = np.abs(np.asarray(host(got), np.float64) - ref)
        ratio[name] = float(np.max(err / (bound + 1e-37))) if err.size else 0.0
        assert (err <= bound + 1e-37).all(), f"{name}: {ratio[name]:.3f} of the bound"

    within("lse", r["lse"], lse, d_lse * has)
    total = loss if reduction == ef.XENT_NONE else np.array([loss.sum() / (max(n, 1) if reduction == ef.XENT_MEAN else 1)])
    d_loss = (d_lse + 4e-6 * np.abs(loss)) * has
    within("loss", r["loss"], total, d_loss if reduction == ef.XENT_NONE else np.array([d_loss.sum() / (max(n, 1) if reduction == ef.XENT_MEAN else 1)]))
    dg = p * (d_lse * np.abs(scale))[:, None] + 4e-6 * np.abs(g)
    if dtype == "bf16":
        dg = dg + 2.0 ** -8 * np.abs(g)
    out = 2.0 ** -8 if dtype == "bf16" else 0.0
    if r["dh"] is not None:
        ref = g @ w.astype(np.float64)
        within("dh", r["dh"], ref, dg @ b + 4e-6 * (np.abs(g) @ b) + out * np.abs(ref))
    if r["dw"] is not None:
        ref = g.T @ np.where(has[:, None], h, 0.0).astype(np.float64)
        within("dw", r["dw"], ref, dg.T @ a + 4e-6 * (np.abs(g).T @ a) + out * np.abs(ref))
    report("xent T=%d V=%d D=%d %s: %s" % (T, V, w.shape[1], dtype, ratio))
    return r


# every tile, whole and ragged: 64 (few tokens), 128, 256; features below and above a stage, whole stages and not
SIZES = [(1, 1, 1), (1, 64, 2), (1, 256, 5000), (2, 63, 65), (64, 64, 64), (65, 65, 255), (63, 200, 4097), (100, 128, 9000), (128, 72, 16500),
         (129, 64, 33000), (300, 128, 8191), (520, 192, 20011), (257, 1088, 700), (1030, 320, 513), (2050, 64, 130), (700, 640, 7000)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,D,V", SIZES)
def test_sizes(T, D, V, dtype):
    check_all(*make(T, D, V, dtype, T + D + V, ignored=0.2 if T > 1 else 0.0), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("reduction", [ef.XENT_NONE, ef.XENT_MEAN, ef.XENT_SUM])
@pytest.mark.parametrize("given", [False, True])
def test_reductions(reduction, given, dtype):
    T = 150
    dloss = None
    if given:
        dloss = np.random.default_rng(9).standard_normal(T if reduction == ef.XENT_NONE else 1)
    check_all(*make(T, 96, 777, dtype, 3, ignored=0.3), dtype, reduction=reduction, dloss=dloss)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tokens_without_a_class_take_no_part(dtype):
    """whatever their features hold; classes outside the vocabulary and the ignored index, which may be a class"""
    h, w, t, hd, wd, td = make(333, 128, 500, dtype, 4)
    t[[0, 7, 100, 200, 332]] = [5, 500, -1, 2 ** 40, 5]
    td = torch.from_numpy(t).cuda()
    out = [i for i in range(333) if t[i] in (5, 500, -1, 2 ** 40)]
    hd[out] = float("nan")
    hd[out[0]] = float("inf")
    r = check_all(h, w, t, hd, wd, td, dtype, ignore=5)
    assert (r["dh"][out] == 0).all() and (r["lse"][out] == 0).all()


@pytest.mark.parametrize("reduction", [ef.XENT_NONE, ef.XENT_MEAN, ef.XENT_SUM])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_token_has_a_class(dtype, reduction):
    h, w, t, hd, wd, td = make(70, 128, 300, dtype, 5)
    td.fill_(-100)
    hd.fill_(float("nan"))
    r = ef.linear_xent_fwd(hd, wd, td, reduction=reduction)
    r.update(ef.linear_xent_bwd(hd, wd, td, r["lse"], reduction=reduction))
    assert all((r[k] == 0).all() for k in ("loss", "lse", "n_valid", "dh", "dw"))


def test_several_pieces_of_the_vocabulary():
    """so many tokens and classes that G is made in pieces, whose last one is ragged and ends inside a stage"""
    for T, V, dtype in ((9000, 15011, "bf16"), (4300, 11000, "f32")):
        h, w, t, hd, wd, td = make(T, 64, V, dtype, 6, ignored=0.5)
        lib = ef.lib()
        code = 1 if dtype == "bf16" else 0
        parts = 1 if dtype == "bf16" else 3
        assert lib.efqat_linear_xent_bwd_workspace_bytes(T, 64, V, code) < 2 * parts * T * V      # the whole of G does not fit it
        check_all(h, w, t, hd, wd, td, dtype)


@pytest.mark.parametrize("T,D,V", [(40, 512, 30000), (300, 128, 40000), (6000, 128, 300), (1500, 256, 1000)])
def test_contractions_in_slices(T, D, V):
    """few results of long contractions: dh over the classes, dw over the tokens"""
    check_all(*make(T, D, V, "bf16", 7), "bf16")
    check_all(*make(T, D, V, "f32", 8, ignored=0.9), "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [128, 100])
def test_rows_that_lie_apart(D, dtype):
    T, V = 200, 900
    h, w, t, hd, wd, td = make(T, D, V, dtype, 10, ignored=0.1)
    big_h, big_w = torch.full((T, D + 56), float("nan"), dtype=hd.dtype, device="cuda"), torch.full((V, D + 24), float("nan"), dtype=hd.dtype, device="cuda")
    hs, ws_ = big_h[:, 8: 8 + D], big_w[:, 16: 16 + D]
    hs.copy_(hd)
    ws_.copy_(wd)
    a = ef.linear_xent_fwd(hd, wd, td)
    a.update(ef.linear_xent_bwd(hd, wd, td, a["lse"]))
    big_dh, big_dw = torch.full((T, D + 3), 7.0, dtype=hd.dtype, device="cuda"), torch.full((V, D + 5), 7.0, dtype=hd.dtype, device="cuda")
    b = ef.linear_xent_fwd(hs, ws_, td)
    b.update(ef.linear_xent_bwd(hs, ws_, td, b["lse"], out=dict(dh=big_dh[:, :D], dw=big_dw[:, :D])))
    assert all(torch.equal(a[k], b[k]) for k in a)
    assert (big_dh[:, D:] == 7.0).all() and (big_dw[:, D:] == 7.0).all()


def test_one_gradient_alone():
    args = make(300, 128, 2000, "bf16", 11)
    both = check_all(*args, "bf16")
    assert torch.equal(check_all(*args, "bf16", want_dw=False)["dh"], both["dh"])
    assert torch.equal(check_all(*args, "bf16", want_dh=False)["dw"], both["dw"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_classes_that_are_masked_out(dtype):
    """logits of the type's lowest magnitude and of minus infinity have no share, and no gradient through it"""
    T, D, V = 90, 64, 400
    h, w, t, hd, wd, td = make(T, D, V, dtype, 12)
    hd[:, 0] = 1.0
    wd[:, 0] = 0.0
    wd[100:200] = 0.0
    wd[100:200, 0] = torch.finfo(hd.dtype).min / 4
    t = np.where((t >= 100) & (t < 200), 5, t)
    td = torch.from_numpy(t).cuda()
    keep = np.r_[0:100, 200:V]
    small = {c: i for i, c in enumerate(keep)}
    r = ef.linear_xent_fwd(hd, wd, td)
    r.update(ef.linear_xent_bwd(hd, wd, td, r["lse"], want_dh=False))
    ts = np.array([small[c] for c in t])
    s = check_all(host(hd).astype(np.float32), host(wd[keep].contiguous()).astype(np.float32), ts, hd, wd[keep].contiguous(), torch.from_numpy(ts).cuda(), dtype)
    assert (r["dw"][100:200] == 0).all()
    assert np.abs(host(r["lse"]) - host(s["lse"])).max() < 1e-5
    wd[100:200, 0] = float("-inf")
    q = ef.linear_xent_fwd(hd, wd, td)
    assert np.abs(host(q["lse"]) - host(s["lse"])).max() < 1e-5 and torch.isfinite(q["loss"]).all()


def test_large_logits():
    """a spread of hundreds: no exponential leaves fp32 in the sums"""
    check_all(*make(130, 64, 3000, "f32", 13, std=20.0), "f32")


def test_a_broken_token_stays_in_its_row_of_dh():
    h, w, t, hd, wd, td = make(100, 64, 300, "bf16", 14)
    hd[17, 3] = float("nan")
    r = ef.linear_xent_fwd(hd, wd, td, reduction=ef.XENT_NONE)
    r.update(ef.linear_xent_bwd(hd, wd, td, r["lse"], reduction=ef.XENT_NONE))
    good = [i for i in range(100) if i != 17]
    assert torch.isnan(r["loss"][17]) and torch.isfinite(r["loss"][good]).all()
    assert torch.isnan(r["dh"][17]).all() and torch.isfinite(r["dh"][good]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_graph_and_stream_and_workspace_contents(dtype):
    T, D, V = 300, 200, 1234
    h, w, t, hd, wd, td = make(T, D, V, dtype, 15, ignored=0.2)
    code = 1 if dtype == "bf16" else 0
    need = max(ef.lib().efqat_linear_xent_fwd_workspace_bytes(T, D, V, code), ef.lib().efqat_linear_xent_bwd_workspace_bytes(T, D, V, code))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    fwd = ef.linear_xent_fwd(hd, wd, td, ws=ws)
    bwd = ef.linear_xent_bwd(hd, wd, td, fwd["lse"], ws=ws)
    ref = [x.clone() for d in (fwd, bwd) for x in d.values()]

    def step():
        ef.linear_xent_fwd(hd, wd, td, ws=ws, out=fwd)
        ef.linear_xent_bwd(hd, wd, td, fwd["lse"], ws=ws, out=bwd)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(3):
        for d in (fwd, bwd):
            for x in d.values():
                x.zero_()
        ws.fill_(255)                                    # NaN in both types
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(ref, (x for d in (fwd, bwd) for x in d.values())):
            assert torch.equal(a, b)


def test_bindings_refuse():
    h, w, t, hd, wd, td = make(8, 64, 16, "bf16", 16)
    lse = torch.zeros(8, device="cuda")
    with pytest.raises(ValueError):
        ef.linear_xent_fwd(hd, wd[:, :32], td)
    with pytest.raises(TypeError):
        ef.linear_xent_fwd(hd, wd.float(), td)
    with pytest.raises(TypeError):
        ef.linear_xent_fwd(hd, wd, td.int())
    with pytest.raises(ValueError):
        ef.linear_xent_fwd(hd, wd, td[:4])
    with pytest.raises(ValueError):
        ef.linear_xent_bwd(hd, wd, td, lse, dloss=torch.ones(8, device="cuda"))
    with pytest.raises(ef.EfqatError):
        ef.linear_xent_bwd(hd, wd, td, lse, want_dh=False, want_dw=False)
    with pytest.raises(ef.EfqatError):
        ef.linear_xent_fwd(hd, wd, td, reduction=3, out=dict(loss=torch.zeros(1, device="cuda")))
    with pytest.raises(ef.EfqatError):
        ef.linear_xent_fwd(hd, wd.new_empty(16 * 64 + 1)[1:].view(16, 64), td)     # whole stages, not aligned to 16 bytes
    with pytest.raises(ef.EfqatError):
        ef.linear_xent_fwd(hd, wd, td, ws=torch.empty(256, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("T", [1024, 1025, 2048, 2049, 4096 + 77, 20000])
def test_the_count_of_tokens(T):
    """tokens counted by one block, by several, by every block for itself"""
    h, w, t, hd, wd, td = make(T, 64, 40, "bf16", T, ignored=0.4)
    t[[0, T - 1]] = [-100, 3]
    r = check_all(h, w, t, hd, wd, torch.from_numpy(t).cuda(), "bf16")
    assert (r["dh"][0] == 0).all() and (r["dh"][T - 1] != 0).any()


@pytest.mark.parametrize("T", [32767, 32768, 133123])
def test_many_tokens(T):
    """as many that the blocks' counts are taken first, and one fewer"""
    h, w, t, hd, wd, td = make(T, 8, 9, "bf16", T, ignored=0.4)
    t[[0, T - 1]] = [-100, 3]
    r = check_all(h, w, t, hd, wd, torch.from_numpy(t).cuda(), "bf16")
    assert (r["dh"][0] == 0).all() and (r["dh"][T - 1] != 0).any()


# logits of few tiles and long rows: their contraction is cut, the softmax follows the join; tiles of 64 and 128, whole and ragged
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,D,V", [(1, 4096, 1), (1, 4096, 3), (5, 3200, 1001), (64, 3136, 64), (70, 4160, 333), (300, 3136, 130), (200, 3500, 999), (700, 3200, 2050)])
def test_contractions_of_logits_in_slices(T, D, V, dtype):
    check_all(*make(T, D, V, dtype, T + D + V, ignored=0.2 if T > 1 else 0.0), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("reduction", [ef.XENT_NONE, ef.XENT_MEAN, ef.XENT_SUM])
def test_reductions_of_logits_in_slices(reduction, dtype):
    h, w, t, hd, wd, td = make(90, 3200, 150, dtype, 7, ignored=0.3)
    rng = np.random.default_rng(8)
    up = rng.standard_normal(90 if reduction == ef.XENT_NONE else 1)
    out = t < 0
    hd[out] = float("nan")
    r = check_all(h, w, t, hd, wd, td, dtype, reduction=reduction, dloss=up)
    assert (r["dh"][torch.from_numpy(out).cuda()] == 0).all()
    td.fill_(-100)
    r = ef.linear_xent_fwd(hd, wd, td, reduction=reduction)
    r.update(ef.linear_xent_bwd(hd, wd, td, r["lse"], reduction=reduction))
    assert all((r[k] == 0).all() for k in ("loss", "lse", "n_valid", "dh", "dw"))


def test_masked_classes_of_logits_in_slices():
    """logits of -inf: no probability, no gradient of their own"""
    h, w, t, hd, wd, td = make(40, 4096, 100, "bf16", 9)
    t[:] = 3 + t % 90
    td = torch.from_numpy(t).cuda()
    hd[:, 0] = 1.0
    wd[:3, 0] = float("-inf")
    r = ef.linear_xent_fwd(hd, wd, td)
    ref = ef.linear_xent_fwd(hd, wd[3:].contiguous(), td - 3)
    assert torch.allclose(r["lse"], ref["lse"], rtol=1e-6, atol=1e-6) and torch.isfinite(r["loss"]).all()
    g = ef.linear_xent_bwd(hd, wd, td, r["lse"])
    assert (g["dw"][:3] == 0).all() and torch.isfinite(g["dw"]).all()


@pytest.mark.parametrize("D,V", [(8, 300), (72, 900), (72, 20011), (520, 20011), (3144, 90)])
@pytest.mark.parametrize("at,ld", [(16, 40), (3, 40), (8, 37)])
def test_classes_as_they_lie(at, ld, D, V):
    """rows of whole 16 bytes that end inside a stage, between NaNs; rows that begin or lie at other addresses"""
    T = 150 if V < 20000 else 600
    h, w, t, hd, wd, td = make(T, D, V, "bf16", D + V + at, ignored=0.1)
    big_w = torch.full((V, D + ld), float("nan"), dtype=wd.dtype, device="cuda")
    ws_ = big_w[:, at: at + D]
    ws_.copy_(wd)
    check_all(h, w, t, hd, ws_, td, "bf16")


@pytest.mark.parametrize("D", [72, 520])
def test_masked_classes_whose_rows_end_inside_a_stage(D):
    h, w, t, hd, wd, td = make(300, D, 20000, "bf16", 12)
    t[:] = 3 + t % 19990
    td = torch.from_numpy(t).cuda()
    hd[:, 0] = 1.0
    wd[:3, 0] = float("-inf")
    r = ef.linear_xent_fwd(hd, wd, td)
    ref = ef.linear_xent_fwd(hd, wd[3:].contiguous(), td - 3)
    assert torch.allclose(r["lse"], ref["lse"], rtol=1e-6, atol=1e-6) and torch.isfinite(r["loss"]).all()
    g = ef.linear_xent_bwd(hd, wd, td, r["lse"])
    assert (g["dw"][:3] == 0).all() and torch.isfinite(g["dw"]).all()


@pytest.mark.parametrize("reduction", [ef.XENT_NONE, ef.XENT_MEAN, ef.XENT_SUM])
@pytest.mark.parametrize("T,V", [(16, 900), (17, 900), (64, 900), (65, 900), (256, 2048), (256, 2049), (257, 2048)])
def test_the_join_of_few_tokens(T, V, reduction):
    """one block that takes 16, 64 or 256 tokens and their mean, or several"""
    check_all(*make(T, 64, V, "bf16", T + V, ignored=0.3), "bf16", reduction=reduction)


@pytest.mark.parametrize("T,D,V,dtype", [(90, 3200, 150, "bf16"), (90, 3200, 150, "f32"), (300, 72, 9000, "bf16"), (700, 640, 7000, "f32"),
                                         (2050, 64, 130, "bf16"), (40, 520, 30000, "bf16"), (33000, 8, 20, "bf16")])
def test_what_the_workspace_held(T, D, V, dtype):
    """NaN in every word of it, in every way that the logits are made: the same bits"""
    h, w, t, hd, wd, td = make(T, D, V, dtype, T + V, ignored=0.3)
    lib, code = ef.lib(), 1 if dtype == "bf16" else 0

    def run(fill):
        ws = [torch.full((n(T, D, V, code),), fill, dtype=torch.uint8, device="cuda")
              for n in (lib.efqat_linear_xent_fwd_workspace_bytes, lib.efqat_linear_xent_bwd_workspace_bytes)]
        r = ef.linear_xent_fwd(hd, wd, td, ws=ws[0])
        r.update(ef.linear_xent_bwd(hd, wd, td, r["lse"], ws=ws[1]))
        return r

    a, b = run(0), run(255)
    assert all(torch.equal(a[k], b[k]) for k in a) and torch.isfinite(b["dw"]).all() and torch.isfinite(b["dh"]).all()


@pytest.mark.parametrize("T,D,V", [(8200, 2112, 520), (1843, 768, 9000), (260, 264, 40000)])
def test_both_products_share_the_blocks(T, D, V):
    """more tiles of dh than blocks; some blocks with slices of dh and the others with dw; few of either"""
    check_all(*make(T, D, V, "bf16", 13, ignored=0.1), "bf16")
