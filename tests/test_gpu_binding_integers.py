"""Integers that a C parameter does not hold are refused, not cut to their lowest 32 bits: a reduction of 2^32 would be taken for 0, losses of
all tokens, in a call that has made room for one."""
import pytest
import torch

import paper_2411_11038_amd as ef

pytestmark = pytest.mark.gpu

WIDE = [2 ** 32, 2 ** 32 + 1, -2 ** 32, 2 ** 31, -2 ** 31 - 1, 2 ** 63]


@pytest.mark.parametrize("n", WIDE)
def test_reduction(n):
    h, w = torch.zeros(8, 64, device="cuda"), torch.zeros(16, 64, device="cuda")
    t, lse = torch.zeros(8, dtype=torch.int64, device="cuda"), torch.zeros(8, device="cuda")
    with pytest.raises(OverflowError):
        ef.linear_xent_fwd(h, w, t, reduction=n)
    with pytest.raises(OverflowError):
        ef.linear_xent_bwd(h, w, t, lse, reduction=n)


@pytest.mark.parametrize("n", WIDE)
def test_kind_and_modes(n):
    x = torch.zeros(4, 16, device="cuda")
    c, s = ef.ckpt8_save(x)
    with pytest.raises(OverflowError):
        ef.act_fwd(x, n)
    with pytest.raises(OverflowError):
        ef.act_bwd(x, n, c, s)
    with pytest.raises(OverflowError):
        ef.fakequant_fwd(x, n, 8, init_minmax=True)
    with pytest.raises(OverflowError):
        ef.fakequant_fwd(x, ef.ACT_PER_TENSOR_ASYM, n, init_minmax=True)


def test_an_index_to_ignore_is_64_bits_wide():
    h, w = torch.randn(8, 64, device="cuda"), torch.randn(16, 64, device="cuda")
    t = torch.arange(8, device="cuda")
    a = ef.linear_xent_fwd(h, w, t, ignore_index=2 ** 40)
    assert int(a["n_valid"]) == 8 and torch.equal(a["loss"], ef.linear_xent_fwd(h, w, t, ignore_index=-2 ** 63)["loss"])
