"""A flag that has no truth value is an error of the call itself: nothing is launched, and the error is the flag's own."""
import numpy as np
import pytest
import torch

import paper_2411_11038_amd as ef

pytestmark = pytest.mark.gpu


class Undecided:
    def __bool__(self):
        raise KeyError("undecided")


@pytest.mark.parametrize("flag,error", [(np.array([True, False]), ValueError), (Undecided(), KeyError)])
def test_checkpoint(flag, error):
    x = torch.ones(4, 16, device="cuda")
    y = torch.full_like(x, 7.0)
    with pytest.raises(error):
        ef.layer_norm_fwd(x, checkpoint=flag, out=dict(y=y))
    with pytest.raises(error):
        ef.act_fwd(x, ef.ACT_GELU, checkpoint=flag, out=dict(y=y))
    assert (y == 7.0).all()
    assert ef.act_fwd(x, ef.ACT_GELU, checkpoint=np.bool_(True))["x_codes"] is not None
    assert ef.act_fwd(x, ef.ACT_GELU, checkpoint=0)["x_codes"] is None
