"""8 bits without inputs (d_in 0): nothing is summed, so z is the bias, and a gradient of the weights has its bias's gradient alone."""
import math

import pytest
import torch

import moe_reference as ref
from test_gpu_moe import TYPES, randn

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


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,k,E,d_z", [(9000, 1, 0, 64), (300, 1, 0, 64), (6000, 2, 3, 24), (40, 2, 3, 24)])
def test_gradient_of_the_bias(gpu_lib, dtype, T, k, E, d_z):
    """db beside a dW without columns, where the rows are taken in parts and where they are not."""
    gen = torch.Generator().manual_seed(T)
    rows, r, parts = T * k, None, [(0, torch.arange(T * k), torch.arange(T * k))]
    if E:
        e = torch.randint(0, E, (T, k), generator=gen, dtype=torch.int32)
        r, parts = gpu_lib.sptir_moe_sort(e.cuda(), E), ref.groups(ref.sort(e, E), k, E, rows, False)
    dZ = randn(gen, rows, d_z, dtype=dtype)
    Q, exponents = torch.empty(rows, 0, dtype=torch.int8, device="cuda"), torch.empty(rows, 0, dtype=torch.uint8, device="cuda")
    dW = torch.empty(max(E, 1), d_z, 0, dtype=dtype, device="cuda")
    db = torch.full((max(E, 1), d_z), math.nan, dtype=dtype, device="cuda")
    gpu_lib.sptir_moe_product_dw_packed(r, dZ.cuda(), Q, exponents, dW, db=db)
    for e, s, _ in parts:
        want = dZ[s].double().sum(0)
        ref.check(db[e], want, ref.bound(want, dZ[s].double().abs().sum(0), len(s), dtype), f"db[{e}]")
