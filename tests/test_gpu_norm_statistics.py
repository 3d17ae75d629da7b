"""Mean and rstd of rows that are not ordinary: they say so, and the rows beside them are what they are without them."""
import numpy as np
import pytest
import torch

import paper_2411_11038_amd as ef

from gpu_util import act_tensor, host

pytestmark = pytest.mark.gpu

# every kernel of the forward: rows shorter than a chunk, in registers (one chunk a lane and two), read again
SIZES = [(6, 5), (6, 300), (6, 1500), (2500, 1024), (6, 9000), (6, 20001)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_rows_that_are_not_finite(rows, cols, dtype):
    a = np.random.default_rng(cols).standard_normal((rows, cols)).astype(np.float32)
    ref = ef.layer_norm_fwd(act_tensor(a, dtype))
    a[0, cols // 2] = np.nan
    a[1, 0] = np.inf
    a[2, cols - 1] = -np.inf
    a[3, 0], a[3, cols - 1] = np.inf, -np.inf
    r = ef.layer_norm_fwd(act_tensor(a, dtype), checkpoint=True)
    mean, rstd = host(r["mean"]), host(r["rstd"])
    assert np.isnan(mean[0]) and mean[1] == np.inf and mean[2] == -np.inf and np.isnan(mean[3])
    assert np.isnan(rstd[:4]).all() and np.isnan(host(r["y"])[:4]).all()
    assert all(torch.equal(r[k][4:], ref[k][4:]) for k in ("y", "mean", "rstd"))
    assert torch.isfinite(r["rstd"][4:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_rows_with_the_lowest_value(rows, cols, dtype):
    """a masked column is finite, its square is not: the statistics and all gradients stay finite"""
    a = np.random.default_rng(cols).standard_normal((rows, cols)).astype(np.float32)
    ref = ef.layer_norm_fwd(act_tensor(a, dtype))
    low = float(torch.finfo(torch.bfloat16 if dtype == "bf16" else torch.float32).min)
    a[0, cols // 2] = a[1, 0] = low
    a[2, cols - 1] = -low
    xd = act_tensor(a, dtype)
    r = ef.layer_norm_fwd(xd, checkpoint=True)
    rstd = host(r["rstd"])
    assert (rstd[:3] >= 0).all() and (rstd[:3] < 1e-18).all()        # the deviation is above 1e38 / sqrt(cols)
    assert all(torch.isfinite(r[k]).all() for k in ("y", "mean"))
    assert np.abs(host(r["mean"])[:3] / (a[:3].astype(np.float64).mean(1)) - 1).max() < 1e-2
    assert all(torch.equal(r[k][3:], ref[k][3:]) for k in ("y", "mean", "rstd"))
    dy = act_tensor(np.ones_like(a), dtype)
    for src in (dict(x=xd), dict(x_codes=r["x_codes"], x_scales=r["x_scales"])):
        o = ef.layer_norm_bwd(dy, None, r["mean"], r["rstd"], **src)
        assert all(torch.isfinite(o[k]).all() for k in o)
