"""Dropout from a counter against its definition: the mask bit for bit, the values rounded once."""
import numpy as np
import pytest
import torch

import paper_2411_11038_amd as ef
from oracle import attn_oracle as ao

from gpu_util import host

pytestmark = pytest.mark.gpu
KINDS = {"bf16": torch.bfloat16, "f32": torch.float32}


def rand(seed, rows, cols, kind, apart=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(rows, cols + apart, generator=g, device="cuda").to(KINDS[kind])[:, :cols]


def state(seed, offset):
    return torch.tensor([seed, offset], dtype=torch.int64, device="cuda")


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,apart", [(1, 1, 0), (3, 7, 2), (5, 64, 0), (130, 33, 1), (2, 2100, 5), (300, 8, 0)])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.999, 1.0])
def test_values(kind, rows, cols, apart, p):
    x, res = rand(1, rows, cols, kind, apart), rand(2, rows, cols, kind, 2 * apart)
    st = state(-1234567890123456789, 2 ** 40 + 3)
    keep, f = ao.dropout_mask(rows, cols, p, -1234567890123456789, 2 ** 40 + 3)
    u = 2.0 ** -8 if kind == "bf16" else 2.0 ** -24
    a, b = host(x).astype(np.float64), host(res).astype(np.float64)
    y = host(ef.dropout_fwd(x, p, st, residual=res)).astype(np.float64)
    ref = b + np.where(keep, a * f, 0.0)
    # the factor and the product are rounded to fp32, the sum once more, then the result
    assert (np.abs(y - ref) <= 1.01 * u * np.abs(ref) + 3 * 2.0 ** -24 * (np.abs(a * f) + np.abs(b))).all() and (y[~keep] == b[~keep]).all()
    d = host(ef.dropout_bwd(x, p, st)).astype(np.float64)
    ref = np.where(keep, a * f, 0.0)
    assert (np.abs(d - ref) <= 1.01 * u * np.abs(ref) + 3 * 2.0 ** -24 * np.abs(ref)).all() and (d[~keep] == 0).all()
    assert (d[keep] != 0).all()


def test_gradient_is_the_slope():
    """linear in x: the backward is the difference of two forwards, exactly where the values are powers of two"""
    x = torch.ones(33, 70, device="cuda")
    st = state(3, 4)
    r = torch.zeros_like(x)
    assert torch.equal(ef.dropout_fwd(2 * x, 0.5, st, residual=r) - ef.dropout_fwd(x, 0.5, st, residual=r), ef.dropout_bwd(x, 0.5, st))


def test_mask_depends_on_place_and_state_alone():
    x = rand(1, 100, 200, "f32")
    one = torch.ones_like(x)
    a = ef.dropout_bwd(one, 0.3, state(1, 2)) != 0
    assert torch.equal(a, ef.dropout_bwd(one.bfloat16(), 0.3, state(1, 2)) != 0)
    wide = torch.ones(100, 333, device="cuda")[:, 5: 205]
    assert torch.equal(a, ef.dropout_bwd(wide, 0.3, state(1, 2)) != 0)
    for other in (state(1, 3), state(2, 2), state(1 + 2 ** 32, 2), state(1, 2 + 2 ** 32)):
        b = ef.dropout_bwd(one, 0.3, other) != 0
        assert abs((a == b).double().mean().item() - 0.58) < 5 * np.sqrt(0.58 * 0.42 / x.numel())     # independent: 0.7^2 + 0.3^2
    for rows, cols in ((100, 200), (1, 20000)):
        m = ef.dropout_bwd(torch.ones(rows, cols, device="cuda"), 0.3, state(7, 7)) != 0
        assert abs(m.double().mean().item() - 0.7) < 5 * np.sqrt(0.21 / m.numel())


def test_in_place_and_what_is_dropped_leaves_nothing():
    x, res, st = rand(1, 40, 100, "bf16"), rand(2, 40, 100, "bf16"), state(9, 9)
    y = ef.dropout_fwd(x, 0.4, st, residual=res)
    a, b = x.clone(), res.clone()
    assert ef.dropout_fwd(a, 0.4, st, residual=res, out=a) is a and torch.equal(a, y)
    ef.dropout_fwd(x, 0.4, st, residual=b, out=b)
    assert torch.equal(b, y)
    gone = ef.dropout_bwd(torch.ones_like(x), 0.4, st) == 0
    for bad in (float("inf"), float("nan")):
        z = ef.dropout_fwd(torch.where(gone, torch.full_like(x, bad), x), 0.4, st, residual=res)
        assert torch.equal(z, y)
        assert torch.equal(ef.dropout_fwd(torch.full_like(x, bad), 1.0, st, residual=res), res)


def test_counter_past_32_bits():
    """chunks are counted in 64 bits: the rows behind chunk 2^32 take other numbers than the first rows (one column a row)"""
    rows = (1 << 32) + 64
    x = torch.ones(1, 1, device="cuda", dtype=torch.bfloat16).expand(rows, 1)       # all rows the same element: stride 0 is refused
    with pytest.raises(ef.EfqatError):
        ef.dropout_bwd(x, 0.5, state(1, 1))
    x = torch.ones(rows, 1, device="cuda", dtype=torch.bfloat16)
    y = ef.dropout_bwd(x, 0.5, state(1, 1), out=x)
    first, last = y[:64, 0].float().cpu().numpy(), y[-64:, 0].float().cpu().numpy()
    for n, got in ((0, first), (1 << 32, last)):
        want = [2.0 if (ao.philox4x32(((n + i) & 0xFFFFFFFF, (n + i) >> 32, 1, 0), (1, 0))[0] & 0xFFFF) >= 32768 else 0.0 for i in range(64)]
        assert got.tolist() == want
    del x, y


def test_captured_graph_draws_anew():
    x, st = torch.ones(64, 512, device="cuda"), state(5, 0)
    y = torch.empty_like(x)
    ef.dropout_fwd(x, 0.5, st, out=y)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ef.dropout_fwd(x, 0.5, st, out=y)
    seen = []
    for step in range(4):
        st[1] = step
        g.replay()
        eager = ef.dropout_fwd(x, 0.5, st)
        torch.cuda.synchronize()
        assert torch.equal(y, eager)
        seen.append(y.clone())
    assert not torch.equal(seen[0], seen[1])


def test_refusals():
    x, st = rand(1, 4, 8, "f32"), state(1, 2)
    for p in (-0.1, 1.5, float("nan")):
        with pytest.raises(ef.EfqatError):
            ef.dropout_fwd(x, p, st)
    with pytest.raises(TypeError):
        ef.dropout_fwd(x, 0.1, st.int())
    with pytest.raises(TypeError):
        ef.dropout_fwd(x, 0.1, None)
    with pytest.raises(TypeError):
        ef.dropout_fwd(x, 0.1, st, residual=x.bfloat16())
    with pytest.raises(ValueError):
        ef.dropout_fwd(x, 0.1, st[:1])
    with pytest.raises(ValueError):
        ef.dropout_fwd(x, 0.1, st, residual=x[:3])
    with pytest.raises(ValueError):
        ef.dropout_fwd(x.cpu(), 0.1, st)
    with pytest.raises(ValueError):
        ef.dropout_fwd(x, 0.1, st.cpu())
