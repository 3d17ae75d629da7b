"""Layer norm of more rows than the chip's blocks take at once, so that each walks several, in both types, with the 8-bit checkpoint and
from it.  Bounds: see test_gpu_norm_act (EPS32 of the terms, and half a unit in the last place of bf16)."""
import numpy as np
import pytest
import torch

import paper_2411_11038_amd as ef
from oracle import lm_oracle as lo

from gpu_util import host
from test_gpu_norm_act import check, check_kept, values

pytestmark = pytest.mark.gpu


# every width class of the kernels: rows by 64 to 1024 lanes, one chunk a lane and two; whole chunks and ragged
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(17003, 64), (9001, 300), (5003, 768), (5003, 777), (4500, 1500), (2100, 3000), (1111, 8192), (600, 9000)])
def test_rows_that_blocks_walk(rows, cols, dtype):
    x, xd = values((rows, cols), dtype, cols, std=1.5)
    dy, dyd = values((rows, cols), dtype, cols + 1)
    w, wd = values((cols,), "f32", cols + 2, std=0.2, mean=1.0)
    b, bd = values((cols,), "f32", cols + 3, std=0.2)
    y, mean, rstd = lo.layer_norm_fwd(x, w, b, 1e-5)
    r = ef.layer_norm_fwd(xd, wd, bd, checkpoint=True)
    check(r["mean"], mean, 6.0, "f32", "mean")
    check(r["rstd"], rstd, 4 * rstd, "f32", "rstd")
    check(r["y"], y, np.abs(y) + 4 * np.abs(w) + np.abs(b), dtype, "y")
    check_kept(r["x_codes"], r["x_scales"], x)
    assert torch.equal(ef.layer_norm_fwd(xd, wd, bd)["y"], r["y"])
    m, s = host(r["mean"]).astype(np.float64), host(r["rstd"]).astype(np.float64)
    for kept in (False, True):
        src = lo.ckpt8_value(*lo.ckpt8(x)) if kept else x.astype(np.float64)
        kw = dict(x_codes=r["x_codes"], x_scales=r["x_scales"]) if kept else dict(x=xd)
        dx, dw, db = lo.layer_norm_bwd(dy, src, m, s, w)
        o = ef.layer_norm_bwd(dyd, wd, r["mean"], r["rstd"], **kw)
        check(o["dx"], dx, 20.0, dtype, "dx")
        check(o["dweight"], dw, (np.abs(dy) * 6).sum(0), "f32", "dweight")
        check(o["dbias"], db, np.abs(dy).astype(np.float64).sum(0), "f32", "dbias")
        again = ef.layer_norm_bwd(dyd, wd, r["mean"], r["rstd"], **kw)
        assert all(torch.equal(o[k], again[k]) for k in o)
