"""8-bit checkpoints of groups that hold the largest finite values of their type (the lowest one is what a mask leaves): they and their
neighbours keep their values, and so do the gradients that are formed from them.

Bounds.  A value read back is one fp32 product, then rounded to the type: equal.  Gradients: EPS32 = 4e-6 (64 roundings of 2^-24) of the
terms they are made of, and 2^-8 of the value more in bf16; the slope of the activation is made of terms of at most 1 + 20."""
import numpy as np
import pytest
import torch

import paper_2411_11038_amd as ef
from oracle import lm_oracle as lo

from gpu_util import act_tensor, host, report

pytestmark = pytest.mark.gpu

EPS32 = 4e-6
KINDS = {"gelu": ef.ACT_GELU, "silu": ef.ACT_SILU}
MOST = {"bf16": float(torch.finfo(torch.bfloat16).max), "f32": float(torch.finfo(torch.float32).max)}


def extremes(cols, dtype, seed):
    """fp32 values that dtype holds; in the first group of the first rows, and in the last, the largest ones"""
    rng = np.random.default_rng(seed)
    x = host(act_tensor(rng.standard_normal((8, cols)).astype(np.float32), dtype)).astype(np.float32)
    top = np.float32(MOST[dtype])
    below = np.float32(127 / 128) * top if dtype == "f32" else np.float32(1.984375 * 2.0 ** 127)   # 128 steps of it still fit fp32
    first = x[:, : min(cols, 128)]
    first[0, 0] = top
    first[1, ::2] = -top                                 # masked columns
    first[2, 0], first[2, -1] = -top, 0.0
    first[3] = top
    first[4, 0] = below
    first[5, 0] = -1.984375 * 2.0 ** 127                # the second largest of bf16
    x[6, cols - 1] = -top
    return x


def check(got, ref, scale, dtype, what):
    got, ref = np.asarray(host(got), np.float64), np.asarray(ref, np.float64)
    assert got.shape == ref.shape and np.isfinite(got).all(), what
    bound = EPS32 * scale + (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 0.0) + 1e-37
    err = np.abs(got - ref)
    report(f"{what}: worst {np.max(err / bound):.3f} of the bound")
    assert (err <= bound).all(), f"{what}: {np.max(err / bound):.3f} of the bound"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [1, 5, 16, 128, 300])
def test_read_back(cols, dtype):
    x = extremes(cols, dtype, cols)
    xd = act_tensor(x, dtype)
    want_codes, want_scales = lo.ckpt8(x)
    want = lo.ckpt8_value(want_codes, want_scales).astype(np.float32)
    assert np.isfinite(want).all()
    kept = [ef.ckpt8_save(xd)]
    r = ef.layer_norm_fwd(xd, checkpoint=True)
    kept.append((r["x_codes"], r["x_scales"]))
    r = ef.act_fwd(xd, ef.ACT_SILU, up=xd, checkpoint=True)
    kept += [(r["x_codes"], r["x_scales"]), (r["up_codes"], r["up_scales"])]
    for codes, scales in kept:
        assert np.array_equal(host(scales), want_scales) and np.array_equal(codes.cpu().numpy()[:, :cols], want_codes)
        assert np.array_equal(host(ef.ckpt8_load(codes, scales, cols, torch.float32)), want)
        if dtype == "bf16":
            assert torch.equal(ef.ckpt8_load(codes, scales, cols, torch.bfloat16), torch.from_numpy(want).cuda().bfloat16())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["gelu", "silu"])
@pytest.mark.parametrize("cols", [5, 300])
def test_activation_gradient(cols, kind, dtype):
    x = extremes(cols, dtype, 1)
    plain = host(act_tensor(np.random.default_rng(2).standard_normal(x.shape).astype(np.float32), dtype)).astype(np.float32)
    dy = host(act_tensor((np.random.default_rng(3).standard_normal(x.shape) * 2.0 ** -20).astype(np.float32), dtype)).astype(np.float32)
    dyd = act_tensor(dy, dtype)

    def kept(a):
        return ef.ckpt8_save(act_tensor(a, dtype)), lo.ckpt8_value(*lo.ckpt8(a))

    for a, b in ((x, None), (x, plain), (plain, x)):
        (ac, as_), ak = kept(a)
        with np.errstate(over="ignore"):
            if b is None:
                dx, _ = lo.act_bwd(dy, ak, kind)
                o = ef.act_bwd(dyd, KINDS[kind], ac, as_)
                up = 1.0
            else:
                (bc, bs), bk = kept(b)
                dx, dup = lo.act_bwd(dy, ak, kind, bk)
                o = ef.act_bwd(dyd, KINDS[kind], ac, as_, bc, bs)
                up = np.abs(bk)
                check(o["dup"], dup, np.abs(dy) * np.where(ak > 20, ak, np.minimum(np.abs(ak), 20) + 1e-3), dtype, "dup")
        check(o["dx"], dx, np.abs(dy) * (1.0 + np.minimum(np.abs(ak), 20)) * up, dtype, "dx")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [5, 300, 9000])
def test_layer_norm_gradient(cols, dtype):
    """rstd as small as the values are large: x rstd is of the order of one"""
    x = extremes(cols, dtype, 4)
    codes, scales = ef.ckpt8_save(act_tensor(x, dtype))
    src = lo.ckpt8_value(*lo.ckpt8(x))
    mean = np.zeros(8)
    rstd = np.array([2.0 ** -126] * 7 + [1.0])
    dy = host(act_tensor((np.random.default_rng(5).standard_normal(x.shape) * 2.0 ** 30).astype(np.float32), dtype)).astype(np.float32)
    w = np.random.default_rng(6).standard_normal(cols).astype(np.float32)
    dx, dw, db = lo.layer_norm_bwd(dy, src, mean, rstd, w)
    f32 = lambda a: torch.from_numpy(np.asarray(a, np.float32)).cuda()
    o = ef.layer_norm_bwd(act_tensor(dy, dtype), f32(w), f32(mean), f32(rstd), x_codes=codes, x_scales=scales)
    xhat = np.abs(src * rstd[:, None])
    g = np.abs(dy * w).astype(np.float64)
    check(o["dx"], dx, rstd[:, None] * (g + g.mean(1, keepdims=True) + xhat * (g * xhat).mean(1, keepdims=True)), dtype, "dx")
    check(o["dweight"], dw, (np.abs(dy) * xhat).sum(0), "f32", "dweight")
    check(o["dbias"], db, np.abs(dy).astype(np.float64).sum(0), "f32", "dbias")
