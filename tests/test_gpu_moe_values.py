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
