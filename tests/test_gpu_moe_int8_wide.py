"""Products of 8-bit integers in tiles of 256 x 256 of which a workgroup has several: a tile's scales change places in LDS with those of the next one,
whose first loads run beside the epilogue that reads the last ones.  Against whole sums on the GPU in 64 bits."""
import math

import pytest
import torch

import moe8_reference as ref8
import moe_reference as ref
import moe_wide_shapes as wide
from test_gpu_moe import TYPES, choices
from test_gpu_moe_wide import near

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,k,E,d_in,d_out,act,dropped", wide.INT8)
def test_product(gpu_lib, dtype, T, k, E, d_in, d_out, act, dropped):
    print("[moe int8 wide]", T, k, E, d_in, d_out, act, dtype, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(T + d_in + d_out)
    rows, n, experts, kept, r = T * k, wide.columns(d_out, act), max(E, 1), T * k, None
    parts = [(0, torch.arange(rows, device="cuda"), torch.arange(rows, device="cuda"))]
    if E:
        e = choices(torch.Generator().manual_seed(T + E), T, k, E, dropped)
        order = ref.sort(e, E)
        r = gpu_lib.sptir_moe_sort(e.cuda(), E)
        parts = [(i, s.cuda(), x.cuda()) for i, s, x in ref.groups(order, k, E, rows, True)]
        kept = int(order[0][-1])

    def whole(*shape):
        return torch.randint(-128, 128, shape, generator=gen, dtype=torch.int8, device="cuda")

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    X, W = whole(T, d_in), whole(experts, n, d_in)
    x_scales, w_scales = torch.exp(normal(T)) / 128, torch.exp(normal(experts, n)) / 128 * d_in ** -0.5
    bias, residual = normal(experts, n).to(dtype), normal(rows, d_out).to(dtype)
    residual[kept:] = math.nan
    for full in (True, False):  # (without what is read beside the sums nothing waits for the next tile's loads)
        y = torch.full((rows, d_out), math.nan, dtype=dtype, device="cuda")
        pre = torch.full((rows, n), math.nan, dtype=dtype, device="cuda") if full else None
        gpu_lib.sptir_moe_product_int8(r, X, x_scales, W, w_scales, y, bias=bias if full else None, residual=residual if full else None, pre=pre,
                                       activation=act, gather=E > 0)
        with torch.device("cuda"):
            want, limit, z, z_limit = ref8.product(parts, rows, X, x_scales, W, w_scales, bias if full else None, residual if full else None, act, dtype)
        near(y, want, limit, "y")
        if full:
            near(pre, z, z_limit, "pre")


@pytest.mark.parametrize("dtype", TYPES)
def test_equal_to_the_kernel_for_few_rows(gpu_lib, dtype):
    """Sums are whole numbers and the rest is float32, row by row: rows of a large call have the bits that they have in a call of their own."""
    rows, d_in, d_out = 3700, 656, 7640
    gen = torch.Generator(device="cuda").manual_seed(1)
    X, W = (torch.randint(-128, 128, (m, d_in), generator=gen, dtype=torch.int8, device="cuda") for m in (rows, d_out))
    x_scales, w_scales = torch.rand(rows, generator=gen, device="cuda"), torch.rand(d_out, generator=gen, device="cuda")
    y, few = torch.empty(rows, d_out, dtype=dtype, device="cuda"), torch.empty(16, d_out, dtype=dtype, device="cuda")
    gpu_lib.sptir_moe_product_int8(None, X, x_scales, W, w_scales, y)
    for first in (0, 1000, 2560, rows - 16):
        gpu_lib.sptir_moe_product_int8(None, X[first:first + 16], x_scales[first:first + 16], W, w_scales, few)
        assert torch.equal(y[first:first + 16], few)
