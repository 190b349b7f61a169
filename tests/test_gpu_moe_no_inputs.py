"""8-bit integers without inputs (d_in 0): nothing is summed, and z is the bias."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,wide", [(500, 24), (20000, 2048)])
@pytest.mark.parametrize("act", ["none", "swiglu"])
def test_product(gpu_lib, rows, wide, act):
    """Whichever kernel takes the call: scales that are no numbers belong to no sum."""
    X, W = torch.empty(rows, 0, dtype=torch.int8, device="cuda"), torch.empty(wide, 0, dtype=torch.int8, device="cuda")
    scales, w_scales = torch.full((rows,), math.nan, device="cuda"), torch.full((wide,), math.inf, device="cuda")
    bias = torch.arange(wide, device="cuda").float().half()
    pre = torch.empty(rows, wide, dtype=torch.float16, device="cuda")
    Y = torch.empty(rows, wide // 2 if act == "swiglu" else wide, dtype=torch.float16, device="cuda")
    gpu_lib.sptir_moe_product_int8(None, X, scales, W, w_scales, Y, bias=bias, pre=pre, activation=act)
    assert torch.equal(pre, bias.expand(rows, wide))
    if act == "none":
        assert torch.equal(Y, bias.expand(rows, wide))
