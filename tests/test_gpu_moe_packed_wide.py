"""dX through a z kept in 8 bits, in tiles of 256 x 256 of which a workgroup has several: codes and exponents of several rows are read at once while the
next tile's first loads run.  Against 64-bit products on what is kept, and bit for bit against the gradient that reads the same values in their type."""
import math

import pytest
import torch

import moe_reference as ref
import moe_wide_shapes as wide
from test_gpu_moe import BF16, F16
from test_gpu_moe_wide import Case, near

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("T,k,E,d_in,d_z,acts,dropped", wide.DX_KEPT)
def test_gradient_of_inputs(gpu_lib, dtype, T, k, E, d_in, d_z, acts, dropped):
    c = Case(gpu_lib, T, k, E, d_in, d_z, dtype, dropped, gather=False)
    dZ, W = c.sorted_rows(d_z), c.tensor(c.E, d_z, d_in, scale=d_z ** -0.5)
    d, size = c.zeros(c.rows, d_in), c.zeros(c.rows, d_in)
    for e, s, _ in c.parts:
        dz, w = dZ[s].double(), W[e].double()
        d[s], size[s] = dz @ w, dz.abs() @ w.abs()
    for act in acts:
        n = wide.columns(d_in, act)
        z = c.tensor(c.rows, n, scale=2.0)
        Q = torch.empty(c.rows, n, dtype=torch.int8, device="cuda")
        exponents = torch.empty(c.rows, -(-n // 32), dtype=torch.uint8, device="cuda")
        gpu_lib.sptir_moe_pack(z, Q, exponents)
        kept = torch.empty_like(z)
        gpu_lib.sptir_moe_unpack(Q, exponents, kept)
        unit = torch.exp2(exponents.double() - 127.0).repeat_interleave(32, 1)[:, :n]
        assert torch.equal(kept.double(), Q.double() * unit)  # (exactly what the codes stand for)
        exponents[c.kept:] = 255                              # rows that belong to no expert reach nothing
        got = torch.full((c.rows, n), math.nan, dtype=dtype, device="cuda")
        gpu_lib.sptir_moe_product_dx_packed(c.r, dZ, W, got, Q, exponents, activation=act)
        plain = torch.full((c.rows, n), math.nan, dtype=dtype, device="cuda")
        gpu_lib.sptir_moe_product_dx(c.r, dZ, W, plain, pre=kept, activation=act)
        assert torch.equal(got, plain), act
        at = c.zeros(c.rows, n)
        at[:c.kept] = kept[:c.kept].double()
        want = ref.slope(d, at, act)
        if act == "swiglu":
            g, u = at.chunk(2, dim=1)
            terms = torch.cat([size * u.abs() * (1.2 + g.abs()), size * (1.0 + g.abs())], 1)
        else:
            terms = size * (1.2 + at.abs())
        near(got, want, ref.bound(want, terms, d_z, dtype), "dX " + act)
