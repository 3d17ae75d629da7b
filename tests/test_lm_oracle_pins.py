"""The fp64 definitions of the operators between the quantized layers against finite differences and closed forms (no GPU)."""
import numpy as np
import pytest

from oracle import lm_oracle as lo


def _differences(f, x, step=1e-5):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        a, b = x.copy(), x.copy()
        a[i] += step
        b[i] -= step
        g[i] = (f(a) - f(b)) / (2 * step)
    return g


def test_checkpoint_codes_and_values():
    x = np.zeros((2, 130), np.float32)
    x[0, :4] = [127.0, -63.5, 0.5, 1.5]                  # scale 1 (or its neighbour): ties go to even
    x[1, 129] = -3e-39                                   # below the smallest scale: codes zero or one step
    codes, scales = lo.ckpt8(x)
    s = np.float32(127.0) * np.float32(1.0 / 127.0)
    assert scales[0, 0] == s and scales[0, 1] == np.float32(2.0 ** -126)
    assert codes[0, 0] == 127 and codes[0, 1] in (-63, -64) and codes[0, 2] in (0, 1) and codes[0, 3] in (1, 2)
    rng = np.random.default_rng(1)
    x = rng.standard_normal((5, 300)).astype(np.float32)
    codes, scales = lo.ckpt8(x)
    step = np.repeat(scales, 128, axis=1)[:, :300].astype(np.float64)
    assert (np.abs(lo.ckpt8_value(codes, scales) - x) <= 0.5001 * step).all()
    x[2, 7] = np.inf
    x[3, 200] = np.nan
    v = lo.ckpt8_value(*lo.ckpt8(x))
    assert np.isnan(v[2, :128]).all() and np.isfinite(v[2, 128:]).all()
    assert np.isnan(v[3, 128:256]).all() and np.isfinite(v[3, :128]).all() and np.isfinite(v[3, 256:]).all()


@pytest.mark.parametrize("kind", ["gelu", "silu"])
@pytest.mark.parametrize("gated", [False, True])
def test_activation_gradient(kind, gated):
    rng = np.random.default_rng(2)
    x, up, dy = (rng.standard_normal((3, 5)) * 2 for _ in range(3))
    u = up if gated else None
    dx, dup = lo.act_bwd(dy, x, kind, u)
    assert np.allclose(dx, _differences(lambda v: (dy * lo.act_fwd(v, kind, u)).sum(), x), atol=1e-8)
    if gated:
        assert np.allclose(dup, _differences(lambda v: (dy * lo.act_fwd(x, kind, v)).sum(), up), atol=1e-8)
    else:
        assert dup is None


def test_layer_norm_gradient():
    rng = np.random.default_rng(3)
    x, dy = rng.standard_normal((4, 6)) + 1.5, rng.standard_normal((4, 6))
    w, b = rng.standard_normal(6), rng.standard_normal(6)
    f = lambda x, w, b: (dy * lo.layer_norm_fwd(x, w, b, 1e-3)[0]).sum()
    y, mean, rstd = lo.layer_norm_fwd(x, w, b, 1e-3)
    dx, dw, db = lo.layer_norm_bwd(dy, x, mean, rstd, w)
    assert np.allclose(dx, _differences(lambda v: f(v, w, b), x), atol=1e-8)
    assert np.allclose(dw, _differences(lambda v: f(x, v, b), w), atol=1e-8)
    assert np.allclose(db, _differences(lambda v: f(x, w, v), b), atol=1e-8)


def test_cross_entropy_gradient():
    rng = np.random.default_rng(4)
    h, w = rng.standard_normal((5, 3)), rng.standard_normal((7, 3))
    t = np.array([0, -100, 6, 7, 2])                     # one ignored, one outside the classes
    scale = rng.standard_normal(5)
    f = lambda h, w: (scale * lo.xent(h, w, t)[0]).sum()
    loss, lse, p, g = lo.xent(h, w, t, dloss=scale)
    assert loss[1] == loss[3] == lse[1] == lse[3] == 0.0 and (g[[1, 3]] == 0).all()
    assert np.allclose(p[[0, 2, 4]].sum(axis=1), 1.0)
    assert np.allclose(g @ w, _differences(lambda v: f(v, w), h), atol=1e-8)
    assert np.allclose(g.T @ h, _differences(lambda v: f(h, v), w), atol=1e-8)
    assert lo.xent(h, w[:1], np.zeros(5, int))[0].max() < 1e-15       # one class: nothing to lose
