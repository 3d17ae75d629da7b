"""Layer norm, the activation of a feed-forward block and the 8-bit checkpoints against the fp64 definitions, at the sizes, strides and
values where they can go wrong.

Bounds.  fp32 results: EPS32 = 4e-6 (64 roundings of 2^-24) of the scale of what is summed; bf16 results: half a unit in the last
place more, at most 2^-8 of the value.  Codes and scales are fp32 operations in a fixed order: equal."""
import numpy as np
import pytest
import torch

import paper_2411_11038_amd as ef
from oracle import lm_oracle as lo

from gpu_util import act_tensor, host, report

pytestmark = pytest.mark.gpu

EPS32 = 4e-6
KINDS = {"gelu": ef.ACT_GELU, "silu": ef.ACT_SILU}
# widths at the ends of chunks, groups and of the kernels' ranges (512, 1024, 2048, 4096, 8192, 16384)
COLS = [1, 7, 8, 127, 128, 129, 136, 512, 513, 1000, 1024, 1025, 2047, 2049, 4096, 4104, 8191, 8200]


def values(shape, dtype, seed, std=1.0, mean=0.0):
    """fp32 values that dtype holds, and their device tensor"""
    a = (np.random.default_rng(seed).standard_normal(shape) * std + mean).astype(np.float32)
    t = act_tensor(a, dtype)
    return host(t).astype(np.float32), t


def apart(t, gap, fill=float("nan")):
    """the same rows, `gap` elements apart, with something else in between"""
    big = torch.full((t.shape[0], t.shape[1] + gap), fill, dtype=t.dtype, device=t.device)
    big[:, : t.shape[1]] = t
    return big[:, : t.shape[1]]


def check(got, ref, scale, dtype, what):
    """scale: of the terms that an element is made of (array or number)"""
    got, ref = np.asarray(host(got), np.float64), np.asarray(ref, np.float64)
    assert got.shape == ref.shape, what
    bound = EPS32 * scale + (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 0.0) + 1e-37
    err = np.abs(got - ref)
    report(f"{what}: worst {np.max(err / bound):.3f} of the bound")
    assert (err <= bound).all(), f"{what}: {np.max(err / bound):.3f} of the bound"


def check_kept(codes, scales, x):
    want_codes, want_scales = lo.ckpt8(x)
    assert np.array_equal(host(scales), want_scales)
    c = codes.cpu().numpy()
    assert np.array_equal(c[:, : x.shape[1]], want_codes) and not c[:, x.shape[1]:].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", COLS + [16384, 16385, 20001])
def test_layer_norm(cols, dtype):
    rows = 37 if cols < 3000 else 5
    x, xd = values((rows, cols), dtype, cols, std=1.5, mean=0.7)
    w, wd = values((cols,), "f32", cols + 1, std=0.3, mean=1.0)
    b, bd = values((cols,), "f32", cols + 2)
    dy, dyd = values((rows, cols), dtype, cols + 3)
    y, mean, rstd = lo.layer_norm_fwd(x, w, b, 1e-5)
    r = ef.layer_norm_fwd(xd, wd, bd, eps=1e-5, checkpoint=True)
    # rstd of one column is 1 / sqrt(eps): differences to the mean are zero but for roundings of x, which it multiplies
    grow = np.abs(x).max() * rstd[:, None] * np.abs(w)
    check(r["mean"], mean, np.abs(x).max(), "f32", "mean")
    check(r["rstd"], rstd, rstd * (1 + (np.abs(x).max() * rstd) ** 2 * 1e-2), "f32", "rstd")
    check(r["y"], y, np.abs(y) + np.abs(b) + grow, dtype, "y")
    check_kept(r["x_codes"], r["x_scales"], x)
    # evaluation: nothing kept
    plain = ef.layer_norm_fwd(xd, wd, bd, eps=1e-5)
    assert torch.equal(plain["y"], r["y"]) and plain["x_codes"] is None
    for kept in (False, True):
        src = lo.ckpt8_value(*lo.ckpt8(x)) if kept else x.astype(np.float64)
        m, s = host(r["mean"]).astype(np.float64), host(r["rstd"]).astype(np.float64)
        dx, dw, db = lo.layer_norm_bwd(dy, src, m, s, w)
        xhat = (src - m[:, None]) * s[:, None]
        kw = dict(x_codes=r["x_codes"], x_scales=r["x_scales"]) if kept else dict(x=xd)
        o = ef.layer_norm_bwd(dyd, wd, r["mean"], r["rstd"], **kw)
        big = np.abs(src).max() * s[:, None]                         # x rstd, before the mean is taken off
        g = np.abs(dy * w)
        terms = s[:, None] * (g + g.mean(1, keepdims=True) + (np.abs(xhat) + big) * (g * (np.abs(xhat) + big)).mean(1, keepdims=True))
        check(o["dx"], dx, terms, dtype, "dx")
        check(o["dweight"], dw, (np.abs(dy) * (np.abs(xhat) + big)).sum(0), "f32", "dweight")
        check(o["dbias"], db, np.abs(dy).sum(0), "f32", "dbias")


@pytest.mark.parametrize("cols", [64, 777, 1500, 3000, 8192, 9000])
def test_layer_norm_many_rows(cols):
    """more rows than the blocks of the chip: each walks several, and their sums are joined"""
    rows = 5003 if cols < 1000 else 1111
    x, xd = values((rows, cols), "f32", 5)
    dy, dyd = values((rows, cols), "f32", 6)
    w, wd = values((cols,), "f32", 7, std=0.2, mean=1.0)
    r = ef.layer_norm_fwd(xd, wd)
    y, mean, rstd = lo.layer_norm_fwd(x, w, 0.0, 1e-5)
    check(r["y"], y, np.abs(y) + 4 * np.abs(w), "f32", "y")
    m, s = host(r["mean"]).astype(np.float64), host(r["rstd"]).astype(np.float64)
    dx, dw, db = lo.layer_norm_bwd(dy, x, m, s, w)
    o = ef.layer_norm_bwd(dyd, wd, r["mean"], r["rstd"], x=xd)
    check(o["dx"], dx, 20.0, "f32", "dx")
    check(o["dweight"], dw, (np.abs(dy) * 6).sum(0), "f32", "dweight")
    check(o["dbias"], db, np.abs(dy).sum(0), "f32", "dbias")
    again = ef.layer_norm_bwd(dyd, wd, r["mean"], r["rstd"], x=xd)
    assert all(torch.equal(o[k], again[k]) for k in o)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gap", [0, 1, 8, 131])
def test_rows_that_lie_apart(dtype, gap):
    rows, cols = 19, 301
    x, xd = values((rows, cols), dtype, 11)
    up, upd = values((rows, cols), dtype, 12)
    dy, dyd = values((rows, cols), dtype, 13)
    w, wd = values((cols,), "f32", 14)
    xs, ups, dys = apart(xd, gap), apart(upd, gap), apart(dyd, gap)
    a, b = ef.layer_norm_fwd(xd, wd, checkpoint=True), ef.layer_norm_fwd(xs, wd, checkpoint=True, out=dict(y=apart(xd, gap, 7.0)))
    assert all(torch.equal(a[k], b[k]) for k in a)
    if gap:
        assert (b["y"].as_strided((rows, gap), (cols + gap, 1), cols) == 7.0).all()
    o = ef.layer_norm_bwd(dyd, wd, a["mean"], a["rstd"], x=xd)
    p = ef.layer_norm_bwd(dys, wd, a["mean"], a["rstd"], x=xs, out=dict(dx=apart(dyd, gap)))
    assert all(torch.equal(o[k], p[k]) for k in o)
    a, b = ef.act_fwd(xd, ef.ACT_SILU, up=upd, checkpoint=True), ef.act_fwd(xs, ef.ACT_SILU, up=ups, checkpoint=True, out=dict(y=apart(xd, gap)))
    assert all(torch.equal(a[k], b[k]) for k in a)
    kept = (a["x_codes"], a["x_scales"], a["up_codes"], a["up_scales"])
    o = ef.act_bwd(dyd, ef.ACT_SILU, *kept)
    p = ef.act_bwd(dys, ef.ACT_SILU, *kept, out=dict(dx=apart(dyd, gap), dup=apart(dyd, gap + 3)))
    assert all(torch.equal(o[k], p[k]) for k in o)
    assert torch.equal(ef.ckpt8_load(*ef.ckpt8_save(xs), cols, xd.dtype), ef.ckpt8_load(*ef.ckpt8_save(xd), cols, xd.dtype, out=apart(xd, gap)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["gelu", "silu"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 4096), (3, 127), (2, 128), (5, 129), (33, 1001), (129, 260), (1, 20001)])
def test_activation(rows, cols, gated, kind, dtype):
    x, xd = values((rows, cols), dtype, 21, std=2.0)
    x[0, 0] = 0.0
    xd[0, 0] = 0.0
    up, upd = values((rows, cols), dtype, 22) if gated else (None, None)
    dy, dyd = values((rows, cols), dtype, 23)
    r = ef.act_fwd(xd, KINDS[kind], up=upd, checkpoint=True)
    u = np.abs(up) if gated else 1.0
    check(r["y"], lo.act_fwd(x, kind, up), (np.abs(x) + 1e-3) * u, dtype, "y")
    check_kept(r["x_codes"], r["x_scales"], x)
    if gated:
        check_kept(r["up_codes"], r["up_scales"], up)
    assert torch.equal(ef.act_fwd(xd, KINDS[kind], up=upd)["y"], r["y"])
    xk = lo.ckpt8_value(*lo.ckpt8(x))
    uk = lo.ckpt8_value(*lo.ckpt8(up)) if gated else None
    dx, dup = lo.act_bwd(dy, xk, kind, uk)
    o = ef.act_bwd(dyd, KINDS[kind], r["x_codes"], r["x_scales"], r["up_codes"], r["up_scales"])
    check(o["dx"], dx, np.abs(dy) * (1.0 + np.abs(xk)) * (np.abs(uk) if gated else 1.0), dtype, "dx")
    if gated:
        check(o["dup"], dup, np.abs(dy) * (np.abs(xk) + 1e-3), dtype, "dup")
    else:
        assert o["dup"] is None


@pytest.mark.parametrize("kind", ["gelu", "silu"])
def test_activation_far_out(kind):
    """values whose exponentials leave fp32: f is 0 or x there, never NaN; an infinity of the right sign stays one"""
    x = np.array([[-3e38, -1e4, -200.0, -90.0, -20.0, 0.0, 20.0, 90.0, 200.0, 1e4, 3e38]], np.float32)
    y = host(ef.act_fwd(act_tensor(x, "f32"), KINDS[kind])["y"])
    assert np.isfinite(y).all() and (y[0, :4] <= 0).all() and (np.abs(y[0, :4]) < 1e-30).all() and np.array_equal(y[0, 7:], x[0, 7:])
    codes, scales = ef.ckpt8_save(act_tensor(np.array([[-1e4, 0.0, 1e4]], np.float32), "f32"))
    dx = host(ef.act_bwd(torch.ones(1, 3, device="cuda"), KINDS[kind], codes, scales)["dx"])
    assert np.abs(dx - np.array([[0.0, 0.5, 1.0]])).max() < 1e-6


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_checkpoint_of_awkward_groups(dtype):
    x, _ = values((6, 400), dtype, 31)
    x[0, 5] = np.inf
    x[1, 200] = np.nan
    x[2, 399] = -np.inf
    x[3] = 0.0
    x[4] = 1e-39 if dtype == "f32" else 0.0
    x[5, :128] = 3e38 if dtype == "f32" else 2.0 ** 127
    xd = act_tensor(x, dtype)
    codes, scales = ef.ckpt8_save(xd)
    v = host(ef.ckpt8_load(codes, scales, 400, torch.float32))
    ref = lo.ckpt8_value(*lo.ckpt8(x))
    assert np.array_equal(np.isnan(v), np.isnan(ref))
    fine = ~np.isnan(ref)
    assert (np.abs(v - ref)[fine] <= 1e-7 * np.abs(ref)[fine]).all()
    # a group that is not finite says so in the gradient of its own columns and nowhere else
    dx = host(ef.act_bwd(torch.ones(6, 400, device="cuda"), ef.ACT_SILU, codes, scales)["dx"])
    assert np.array_equal(np.isnan(dx), np.isnan(ref))


def test_layer_norm_keeps_a_broken_row_to_itself():
    x, xd = values((9, 1500), "f32", 41)
    xd[4, 700] = float("nan")
    xd[6, 1] = float("inf")
    r = ef.layer_norm_fwd(xd, checkpoint=True)
    good = [0, 1, 2, 3, 5, 7, 8]
    y, mean, rstd = lo.layer_norm_fwd(x[good], 1.0, 0.0, 1e-5)
    check(r["y"][good], y, np.abs(y) + 4, "f32", "y")
    assert torch.isnan(r["y"][4]).all() and torch.isnan(r["y"][6]).any()
    o = ef.layer_norm_bwd(torch.ones_like(xd), None, r["mean"], r["rstd"], x=xd)
    assert torch.isfinite(o["dx"][good]).all() and torch.isnan(o["dx"][4]).all()


def test_layer_norm_of_an_offset_row():
    """an offset of a thousand deviations costs the digits of x itself, no more"""
    x = (np.random.default_rng(42).standard_normal((4, 4096)) + 1000.0).astype(np.float32)
    y, mean, rstd = lo.layer_norm_fwd(x, 1.0, 0.0, 1e-5)
    r = ef.layer_norm_fwd(torch.from_numpy(x).cuda())
    assert np.abs(host(r["mean"]) - mean).max() <= 2.0 ** -14          # an ulp of 1000 in fp32 is 2^-14
    assert np.abs(host(r["rstd"]) / rstd - 1).max() <= 1e-6
    assert np.abs(host(r["y"]) - y).max() <= 2.0 ** -13


def test_offsets_beyond_32_bits():
    """rows that lie 2^31 elements apart"""
    ld, cols = 2 ** 31 + 24, 200
    big = torch.empty(ld + cols, dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((2, cols), (ld, 1))
    src, srcd = values((2, cols), "bf16", 51)
    x.copy_(srcd)
    a, b = ef.layer_norm_fwd(srcd, checkpoint=True), ef.layer_norm_fwd(x, checkpoint=True)
    assert all(torch.equal(a[k], b[k]) for k in a)
    c, d = ef.act_fwd(srcd, ef.ACT_GELU, checkpoint=True), ef.act_fwd(x, ef.ACT_GELU, checkpoint=True)
    assert all(c[k] is None or torch.equal(c[k], d[k]) for k in c)
    assert torch.equal(ef.layer_norm_bwd(srcd, None, a["mean"], a["rstd"], x=srcd)["dx"],
                       ef.layer_norm_bwd(srcd, None, a["mean"], a["rstd"], x=x)["dx"])


def test_graph_and_stream_and_workspace_contents():
    rows, cols = 700, 1032
    x, xd = values((rows, cols), "bf16", 61)
    dy, dyd = values((rows, cols), "bf16", 62)
    w, wd = values((cols,), "f32", 63)
    need = ef.lib().efqat_layer_norm_bwd_workspace_bytes(rows, cols)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    fwd, bwd = ef.layer_norm_fwd(xd, wd, checkpoint=True), None
    bwd = ef.layer_norm_bwd(dyd, wd, fwd["mean"], fwd["rstd"], x_codes=fwd["x_codes"], x_scales=fwd["x_scales"], ws=ws)
    act = ef.act_fwd(xd, ef.ACT_GELU, up=dyd, checkpoint=True)
    dact = ef.act_bwd(dyd, ef.ACT_GELU, act["x_codes"], act["x_scales"], act["up_codes"], act["up_scales"])
    ref = [t.clone() for d in (fwd, bwd, act, dact) for t in d.values()]

    def step():
        ef.layer_norm_fwd(xd, wd, checkpoint=True, out=fwd)
        ef.layer_norm_bwd(dyd, wd, fwd["mean"], fwd["rstd"], x_codes=fwd["x_codes"], x_scales=fwd["x_scales"], ws=ws, out=bwd)
        ef.act_fwd(xd, ef.ACT_GELU, up=dyd, checkpoint=True, out=act)
        ef.act_bwd(dyd, ef.ACT_GELU, act["x_codes"], act["x_scales"], act["up_codes"], act["up_scales"], out=dact)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(3):
        for d in (fwd, bwd, act, dact):
            for t in d.values():
                t.zero_()
        ws.fill_(255)                                    # NaN, as fp32: nothing is read that the call did not write
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(ref, (t for d in (fwd, bwd, act, dact) for t in d.values())):
            assert torch.equal(a, b)


def test_bindings_refuse():
    x = torch.zeros(4, 16, device="cuda")
    c, s = ef.ckpt8_save(x)
    with pytest.raises(ValueError):
        ef.ckpt8_save(x.t())                             # columns that lie apart
    with pytest.raises(ValueError):
        ef.layer_norm_fwd(x[0])
    with pytest.raises(ValueError):
        ef.act_fwd(x.cpu(), ef.ACT_GELU)
    with pytest.raises(TypeError):
        ef.act_fwd(x.half(), ef.ACT_GELU)
    with pytest.raises(TypeError):
        ef.act_fwd(x, ef.ACT_GELU, up=x.bfloat16())
    with pytest.raises(ValueError):
        ef.act_bwd(x, ef.ACT_GELU, c[:2], s)
    with pytest.raises(ValueError):
        ef.act_bwd(x, ef.ACT_GELU, c, s, up_codes=c)
    with pytest.raises(ValueError):
        ef.layer_norm_bwd(x, None, x[:, 0].contiguous(), x[:, 0].contiguous())
    with pytest.raises(TypeError):
        ef.layer_norm_fwd(x, weight=torch.ones(16, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        ef.layer_norm_fwd(x, weight=torch.ones(15, device="cuda"))
    with pytest.raises(ef.EfqatError):
        ef.act_fwd(x, 9)
    with pytest.raises(ef.EfqatError):
        ef.layer_norm_fwd(torch.zeros(0, 16, device="cuda"))
    with pytest.raises(ef.EfqatError):
        ef.layer_norm_fwd(x, eps=-1.0)
