"""Activations where their values are small, and at the ends of the types.  z comes from the bias alone: x is zero."""
import math

import pytest
import torch

import moe_reference as ref
from test_gpu_moe import ACTS, TYPES, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [3, 300])
def test_gelu_keeps_its_digits_in_single_precision(gpu_lib, rows):
    """Below -4 the normal distribution function is too small for 1 + erf: that has no digit left at -5.5."""
    z = torch.cat([torch.linspace(-12.5, 6.0, 1021), torch.tensor([0.0, -0.0, 1e-30, -1e-30])])
    y = torch.empty(rows, len(z), device="cuda")
    gpu_lib.sptir_moe_product(None, torch.zeros(rows, 8, device="cuda"), torch.ones(len(z), 8, device="cuda"), y, bias=z.cuda(), activation="gelu")
    want = (0.5 * z.double() * torch.erfc(-z.double() / math.sqrt(2.0)))[None]
    # erfc(x) moves by 2 x^2 + 1 times the relative error of x (1.5 roundings); 24 roundings for the functions and products
    limit = want.abs() * 2.0 ** -24 * (1.5 * z.double() ** 2 + 24.0) + 1e-44
    for i in range(0, rows, 99):
        ref.check(y[i:i + 1], want, limit, "y")


def ends(dtype):
    info = torch.finfo(dtype)
    v = [0.0, -0.0, info.tiny, -info.tiny, 1.0, -1.0, 5.5, -5.5, 30.0, -30.0, 104.0, -104.0, 6e4, -6e4, info.max, info.min, math.nan]
    return torch.tensor(v, dtype=torch.float64).to(dtype)


def check_ends(got, want, limit, what):
    """What the type cannot hold (2 * 65,504 of float16) is an infinity."""
    over = want.abs() > torch.finfo(got.dtype).max
    beyond = got.cpu().double()[over]
    assert bool(torch.isinf(beyond).all()) and torch.equal(torch.sign(beyond), torch.sign(want[over])), what
    ref.check(torch.where(over.to(got.device), 0.0, got.double()), torch.where(over, 0.0, want), limit, what)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("rows,d_in", [(3, 64), (3, 7), (300, 64), (300, 7)])
def test_activation_at_the_ends(gpu_lib, dtype, act, rows, d_in):
    """The lowest and the largest value, signed zeros, tiny values, and NaN, which no activation may hide (torch's do not)."""
    say("ends", dtype, act, rows, d_in)
    v = ends(dtype)
    if act == "swiglu":  # every gate with every moderate value beside it
        other = torch.tensor([1.0, -0.5, math.nan], dtype=dtype)
        z = torch.cat([v.repeat_interleave(3), other.repeat(len(v))])
    else:
        z = v
    X, W = torch.zeros(rows, d_in, dtype=dtype, device="cuda"), torch.ones(len(z), d_in, dtype=dtype, device="cuda")
    want = ref.activation(z.double()[None], act)
    y, pre = (torch.empty(rows, n, dtype=dtype, device="cuda") for n in (want.shape[1], len(z)))
    gpu_lib.sptir_moe_product(None, X, W, y, bias=z.cuda(), activation=act, pre=pre)
    # 16 roundings of float32 of the value, as wide as a few units of the exponent's argument at 104 (that is 2^-24 * 104 relative)
    limit = ref.bound(want, want.abs() * 8, 1, dtype) + 1e-36
    for i in range(0, rows, 99):
        check_ends(y[i:i + 1], want, limit, "y")
    assert torch.equal(torch.nan_to_num(pre.cpu(), 9.0), torch.nan_to_num(z[None].expand(rows, -1), 9.0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ACTS[1:])
@pytest.mark.parametrize("width", [0, 3])
def test_derivative_at_the_ends(gpu_lib, dtype, act, width):
    say("derivative at the ends", dtype, act, width)
    v = ends(dtype)
    v = torch.cat([v, v[:7], torch.ones(width, dtype=dtype)])  # (24: whole words; and not)
    n, rows = len(v), 5
    pre = v[None].expand(rows, -1)
    if act == "swiglu":
        pre = torch.cat([pre, torch.tensor([1.0, -0.5, 2.0, math.nan, 1.0], dtype=dtype)[:, None].expand(-1, n)], 1)
    d = torch.tensor([1.0, -2.0, 0.5, 1.0, 0.25], dtype=dtype)[:, None].expand(-1, n)
    # dX = dZ times the identity
    eye = torch.eye(n, dtype=dtype, device="cuda")
    got = torch.empty(pre.shape, dtype=dtype, device="cuda")
    gpu_lib.sptir_moe_product_dx(None, d.contiguous().cuda(), eye, got, pre=pre.contiguous().cuda(), activation=act)
    want = ref.slope(d.double(), pre.double(), act)
    # the slope's terms: up to |z| near 1, and what is left of them where the exponential is below 2^-24
    limit = ref.bound(want, d.double().abs().repeat(1, want.shape[1] // n) * 8, 1, dtype) + want.abs() * 2.0 ** -20
    check_ends(got, want, limit, "dX")
