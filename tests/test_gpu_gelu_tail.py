"""GELU and SiLU of negative values, whose results are small: they keep their relative accuracy.

Bounds, relative to the value (the slope: to the two terms that it is made of): 16 roundings of 2^-24 = 2^-20 in fp32 (the fitted tail 1.5,
its evaluation with reciprocal and exponential up to 10, products 3); bf16: the rounding of the exponential's argument, 2^-24 x^2 / 2, and half
a unit in the last place, at most 2^-8, more.  SiLU: 6 roundings and the argument's and its factor's, |x| each."""
import math

import numpy as np
import pytest
import torch

import paper_2411_11038_amd as ef
from oracle import lm_oracle as lo

from gpu_util import act_tensor, host, report

pytestmark = pytest.mark.gpu

_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def phi(x):
    return 0.5 * _erfc(-x / math.sqrt(2.0))


def gauss(x):
    return np.exp(-0.5 * x * x) / math.sqrt(2.0 * math.pi)


def kept(a):
    """what the checkpoint of a stands for: a product in fp32 (at x = -12.5 a rounding of x is 156 of its tail)"""
    return lo.ckpt8_value(*lo.ckpt8(a)).astype(np.float32).astype(np.float64)


def check(got, ref, terms, x, dtype, what):
    bound = 2.0 ** -20 * terms
    if dtype == "bf16":
        bound = bound + 2.0 ** -24 * 0.5 * x * x * terms + 2.0 ** -8 * np.abs(ref)
    err = np.abs(np.asarray(host(got), np.float64) - ref)
    report(f"{what}: worst {np.max(err / (bound + 1e-300)):.3f} of the bound")
    assert (err <= bound).all(), what


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [4096, 1001, 7])
def test_value(cols, dtype):
    a = np.stack([np.linspace(-12.5, -0.01, cols), np.linspace(-4.0, -1.0, cols), np.linspace(0.01, 12.5, cols)]).astype(np.float32)
    xd = act_tensor(a, dtype)
    x = host(xd).astype(np.float64)
    ref = x * phi(x)
    check(ef.act_fwd(xd, ef.ACT_GELU)["y"], ref, np.abs(ref), x, dtype, "value")
    up = act_tensor(np.full_like(a, 2.0), dtype)
    check(ef.act_fwd(xd, ef.ACT_GELU, up=up)["y"], 2 * ref, 2 * np.abs(ref), x, dtype, "gated value")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_value_of_silu(dtype):
    xd = act_tensor(np.linspace(-80.0, -0.01, 5000)[None].astype(np.float32), dtype)
    x = host(xd).astype(np.float64)
    ref = x / (1.0 + np.exp(-x))
    bound = (2.0 ** -24 * (6 + 2 * np.abs(x)) + (2.0 ** -8 if dtype == "bf16" else 0.0)) * np.abs(ref)
    err = np.abs(np.asarray(host(ef.act_fwd(xd, ef.ACT_SILU)["y"]), np.float64) - ref)
    report(f"silu: worst {np.max(err / bound):.3f} of the bound")
    assert (err <= bound).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lowest", [-12.5, -8.0, -3.0, -1.0, 6.0])
def test_slope(lowest, dtype):
    a = np.tile(np.linspace(lowest, 0.0, 128), (2, 3)).astype(np.float32)
    x = kept(a)
    codes, scales = ef.ckpt8_save(torch.from_numpy(a).cuda())
    ones = act_tensor(np.ones_like(a), dtype)
    o = ef.act_bwd(ones, ef.ACT_GELU, codes, scales)
    check(o["dx"], phi(x) + x * gauss(x), phi(x) + np.abs(x) * gauss(x), x, dtype, "slope")
    uc, us = ef.ckpt8_save(torch.full_like(torch.from_numpy(a), 2.0).cuda())
    u = kept(np.full_like(a, 2.0))
    o = ef.act_bwd(ones, ef.ACT_GELU, codes, scales, uc, us)
    check(o["dx"], (phi(x) + x * gauss(x)) * u, (phi(x) + np.abs(x) * gauss(x)) * u, x, dtype, "gated slope")
    check(o["dup"], x * phi(x), np.abs(x * phi(x)), x, dtype, "gradient of the gate")
