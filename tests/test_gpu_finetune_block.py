"""The example that trains a feed-forward block with its norms, head and loss: it learns, and its gradients are those of the loss."""
import numpy as np
import pytest
import torch

from oracle import lm_oracle as lo
from workloads import finetune_block as fb

from gpu_util import host

pytestmark = pytest.mark.gpu


def test_the_block_learns():
    m, x, targets = fb.make(192, 128, 344, 97)
    first = fb.step(m, x, targets)
    assert abs(float(first["loss"]) - np.log(97)) < 0.3 and int(first["n_valid"]) == int((targets >= 0).sum())
    for _ in range(40):
        last = fb.step(m, x, targets, lr=0.5)
    assert float(last["loss"]) < 0.5 * float(first["loss"])
    assert all(torch.isfinite(t).all() for t in (last["dx"], last["dhead"], m.w1, m.w2, m.head))


def test_the_head_and_last_norm_get_the_gradient_of_the_loss():
    """against the fp64 definitions, from the same input of the last norm: its 8 bits are what the gradient is taken at"""
    m, x, targets = fb.make(100, 64, 176, 53, seed=3)
    m.w2.zero_()                                         # the block adds nothing: the last norm sees x
    head, w = host(m.head.bfloat16()), host(m.norm[1][0])
    r = fb.step(m, x, targets, lr=0.0)
    xs = host(x)
    t = targets.cpu().numpy()
    n = int((t >= 0).sum())
    y, mean, rstd = lo.layer_norm_fwd(xs, w, 0.0, 1e-5)
    loss, _, _, g = lo.xent(y, head, t, dloss=np.full(100, 1.0 / n))
    assert abs(float(r["loss"]) - loss.sum() / n) < 0.01 * abs(loss.sum() / n)
    kept = lo.ckpt8_value(*lo.ckpt8(xs.astype(np.float32)))
    _, dw, db = lo.layer_norm_bwd(g @ head, kept, mean, rstd, w)
    # the norm's output, G and dh are rounded to bf16 (2^-9 of each term in the mean, 100 terms a sum)
    for got, ref in ((r["norms"][1]["dweight"], dw), (r["norms"][1]["dbias"], db), (r["dhead"], g.T @ y)):
        assert np.linalg.norm(host(got) - ref) <= 0.02 * np.linalg.norm(ref)
