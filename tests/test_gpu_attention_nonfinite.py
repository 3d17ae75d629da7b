"""What is not finite in a query or an upstream gradient stays in its sequence and key head: the gradients of all others are as without it."""
import pytest
import torch

import paper_2411_11038_amd as ef

pytestmark = pytest.mark.gpu
KINDS = {"bf16": torch.bfloat16, "f32": torch.float32}


def rand(seed, rows, cols, kind):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(rows, cols, generator=g, device="cuda").to(KINDS[kind])


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 2)])
def test_queries_and_upstream_gradients(kind, dim, value, window, sinks):
    heads, kv, start = 4, 2, torch.tensor([0, 50, 110], dtype=torch.int32, device="cuda")
    q, k, v, do = rand(1, 110, heads * dim, kind), rand(2, 110, kv * dim, kind), rand(3, 110, kv * dim, kind), rand(4, 110, heads * dim, kind)
    how = dict(kv_heads=kv, q_start=start, window=window, sinks=sinks)

    def run():
        r = ef.attention_fwd(q, k, v, heads, **how)
        return r, ef.attention_bwd(do, q, k, v, r["o"], r["lse"], heads, **how)
    r, g = run()
    q[20, 5] = float("nan")                                  # sequence 0, head 0: key head 0
    do[70, 3 * dim + 1] = value                              # sequence 1, head 3: key head 1
    r2, g2 = run()

    def apart(t, u, *spoilt):
        keep = torch.ones(t.shape, dtype=torch.bool, device="cuda")
        for rows, cols in spoilt:
            keep[rows, cols] = False
        return torch.equal(t[keep], u[keep])
    assert apart(r["o"], r2["o"], (slice(20, 21), slice(0, dim)))            # a query is its token's alone
    assert apart(r["lse"].t(), r2["lse"].t(), (slice(20, 21), slice(0, 1)))
    assert apart(g["dq"], g2["dq"], (slice(20, 21), slice(0, dim)), (slice(70, 71), slice(3 * dim, 4 * dim)))
    for name in ("dk", "dv"):
        assert apart(g[name], g2[name], (slice(0, 50), slice(0, dim)), (slice(50, 110), slice(dim, 2 * dim))), name
    assert not torch.isfinite(r2["o"][20, :dim].float()).all() and not torch.isfinite(g2["dq"][70, 3 * dim:].float()).all()
