"""Products in tiles of 256 x 256 of which a workgroup has several: the next tile's first loads run beside the last one's epilogue.
Against 64-bit products on the same inputs, with the error that moe_reference.bound allows."""
import math

import pytest
import torch

import moe_reference as ref
import moe_wide_shapes as wide
from test_gpu_moe import BF16, F16, choices

pytestmark = pytest.mark.gpu


def near(got, want, limit, what):
    over = (got.double() - want).abs() - limit
    assert not bool(torch.isnan(over).any()), f"{what}: NaN"
    assert float(over.max()) <= 0.0, f"{what}: {int((over > 0).sum())} of {over.numel()} places off"


class Case:
    def __init__(self, lib, T, k, E, d_in, d_z, dtype, dropped, gather):
        print("[moe wide]", T, k, E, d_in, d_z, dtype, dropped, gather, flush=True)
        self.lib, self.T, self.k, self.E, self.dtype = lib, T, k, max(E, 1), dtype
        self.gen = torch.Generator(device="cuda").manual_seed(T + d_in + d_z)
        self.rows, self.r = T * k, None
        self.parts = [(0, torch.arange(self.rows, device="cuda"), torch.arange(self.rows, device="cuda"))]
        self.kept = self.rows
        if E:
            e = choices(torch.Generator().manual_seed(T + E), T, k, E, dropped)
            order = ref.sort(e, E)
            self.r = lib.sptir_moe_sort(e.cuda(), E)
            self.parts = [(i, s.cuda(), x.cuda()) for i, s, x in ref.groups(order, k, E, self.rows, gather)]
            self.kept = int(order[0][-1])

    def tensor(self, *shape, scale=1.0):
        return (torch.randn(*shape, generator=self.gen, device="cuda") * scale).to(self.dtype)

    def sorted_rows(self, cols):
        t = self.tensor(self.rows, cols)
        t[self.kept:] = math.nan  # rows that belong to no expert reach nothing
        return t

    def zeros(self, *shape):
        return torch.zeros(*shape, dtype=torch.float64, device="cuda")


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("T,k,E,d_in,d_out,act,dropped", wide.FORWARD)
def test_forward(gpu_lib, dtype, T, k, E, d_in, d_out, act, dropped):
    n = wide.columns(d_out, act)
    c = Case(gpu_lib, T, k, E, d_in, n, dtype, dropped, gather=E > 0)
    X, W, bias = c.tensor(T if E else c.rows, d_in), c.tensor(c.E, n, d_in, scale=d_in ** -0.5), c.tensor(c.E, n)
    residual = c.sorted_rows(d_out)
    z, size, r = c.zeros(c.rows, n), c.zeros(c.rows, n), c.zeros(c.rows, d_out)
    plain = c.zeros(c.rows, n)
    for e, s, x in c.parts:
        a, w = X[x].double(), W[e].double()
        plain[s] = a @ w.t().contiguous()
        z[s] = plain[s] + bias[e].double()
        size[s] = a.abs() @ w.abs().t().contiguous() + bias[e].double().abs()
        r[s] = residual[s].double()
    for full in (True, False):  # (without what is read beside the sums nothing waits for the next tile's loads)
        y = torch.full((c.rows, d_out), math.nan, dtype=dtype, device="cuda")
        pre = torch.full((c.rows, n), math.nan, dtype=dtype, device="cuda") if full else None
        gpu_lib.sptir_moe_product(c.r, X, W, y, bias=bias if full else None, residual=residual if full else None, pre=pre,
                                  activation=act, gather=E > 0)
        at = z if full else plain
        want = ref.activation(at, act)
        if act == "swiglu":
            g, u = at.chunk(2, dim=1)
            sg, su = size.chunk(2, dim=1)
            terms = 1.2 * sg * u.abs() + ref.activation(g, "silu").abs() * su + want.abs() + sg * su * 4.0 * (math.sqrt(d_in) + 8.0) * 2.0 ** -24
        else:
            terms = 1.2 * size
        if full:
            want, terms = want + r, terms + r.abs()
            near(pre, z, ref.bound(z, size, d_in, dtype), "pre")
        near(y, want, ref.bound(want, terms, d_in, dtype), "y")


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("T,k,E,d_in,d_out,act,dropped", wide.DX)
def test_gradient_of_inputs(gpu_lib, dtype, T, k, E, d_in, d_out, act, dropped):
    c = Case(gpu_lib, T, k, E, d_in, d_out, dtype, dropped, gather=False)
    dZ, W = c.sorted_rows(d_out), c.tensor(c.E, d_out, d_in, scale=d_out ** -0.5)
    d, size = c.zeros(c.rows, d_in), c.zeros(c.rows, d_in)
    for e, s, _ in c.parts:
        dz, w = dZ[s].double(), W[e].double()
        d[s], size[s] = dz @ w, dz.abs() @ w.abs()
    for act in {act, "none"}:
        n = wide.columns(d_in, act)
        pre = c.sorted_rows(n) if act != "none" else None
        got = torch.full((c.rows, n), math.nan, dtype=dtype, device="cuda")
        gpu_lib.sptir_moe_product_dx(c.r, dZ, W, got, pre=pre, activation=act)
        want, terms = d, size
        if act != "none":
            at = c.zeros(c.rows, n)
            at[:c.kept] = pre[:c.kept].double()
            want = ref.slope(d, at, act)
            if act == "swiglu":
                g, u = at.chunk(2, dim=1)
                terms = torch.cat([size * u.abs() * (1.2 + g.abs()), size * (1.0 + g.abs())], 1)
            else:
                terms = size * (1.2 + at.abs())
        near(got, want, ref.bound(want, terms, d_out, dtype), "dX " + act)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("T,k,E,d_in,d_out,dropped", wide.DW)
def test_gradient_of_weights(gpu_lib, dtype, T, k, E, d_in, d_out, dropped):
    c = Case(gpu_lib, T, k, E, d_in, d_out, dtype, dropped, gather=E > 0)
    X, dZ = c.tensor(T if E else c.rows, d_in), c.sorted_rows(d_out)
    for with_db in (True, False):
        dW = torch.full((c.E, d_out, d_in), math.nan, dtype=dtype, device="cuda")
        db = torch.full((c.E, d_out), math.nan, dtype=dtype, device="cuda") if with_db else None
        gpu_lib.sptir_moe_product_dw(c.r, dZ, X, dW, db=db, gather=E > 0)
        most = max(len(s) for _, s, _ in c.parts)
        for e, s, x in c.parts:
            a, dz = X[x].double(), dZ[s].double()
            across = dz.t().contiguous()
            want = across @ a
            near(dW[e], want, ref.bound(want, across.abs() @ a.abs(), most, dtype), f"dW[{e}]")
            if with_db:
                want = dz.sum(0)
                near(db[e], want, ref.bound(want, dz.abs().sum(0), most, dtype), f"db[{e}]")
