"""The same operators where another kernel, tile or split takes the call: large tiles beside small ones, weight gradients whose
rows are taken in parts, many experts, rows of a whole workgroup, matrices that experts share."""
import ctypes
import math

import pytest
import torch

import moe_reference as ref
from paper_2207_04606_amd import moe
from test_gpu_moe import BF16, F16, F32, TYPES, Case, choices, out_like, randn, say

pytestmark = pytest.mark.gpu
HALF = [F16, BF16]


# few tiles and many rows; parts that end inside a step; experts of very different sizes, one without rows
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,k,E,d_in,d_out,dropped", [(9000, 1, 0, 40, 24, 0.0), (20011, 1, 0, 130, 71, 0.0), (6000, 2, 3, 64, 96, 0.2),
                                                      (4096, 1, 0, 256, 520, 0.0), (7001, 1, 5, 72, 8, 0.0), (4100, 1, 0, 3, 1, 0.0)])
def test_weight_gradient_of_many_rows(gpu_lib, dtype, T, k, E, d_in, d_out, dropped):
    c = Case(gpu_lib, T, k, E, d_in, d_out, dtype, dropped=dropped)
    assert moe._library().sptir_moe_product_dw_workspace(c.rows, c.E, d_in, d_out) > 0
    c.dw()
    c.dw(db=False)
    first, again = (torch.empty(c.E, d_out, d_in, dtype=dtype, device="cuda") for _ in range(2))
    for dW in (first, again):
        gpu_lib.sptir_moe_product_dw(c.r, c.dZ_dev, c.X_dev, dW, gather=c.gather)
    assert torch.equal(first, again)
    c = Case(gpu_lib, T, k, E, d_in, d_out, dtype, dropped=dropped, gather=False, extra=3)
    c.dw()


@pytest.mark.parametrize("dtype", TYPES)
def test_weight_gradient_without_inputs(gpu_lib, dtype):
    """Nothing but the sums of dZ, in one part and in several; an expert without rows has zeros."""
    for T, k, E, d_z in ((50, 2, 4, 24), (9000, 1, 0, 100), (8000, 1, 3, 17)):
        gen = torch.Generator().manual_seed(T)
        routing, ptr = None, torch.tensor([0, T * k])
        if E:
            e = choices(gen, T, k, E)
            e[e == 1] = 0
            routing, ptr = gpu_lib.sptir_moe_sort(e.cuda(), E), ref.sort(e, E)[0].long()
        dZ = randn(gen, T * k, d_z, dtype=dtype)
        db = torch.full((max(E, 1), d_z), math.nan, dtype=dtype, device="cuda")
        gpu_lib.sptir_moe_product_dw(routing, dZ.cuda(), torch.empty(T * k, 0, dtype=dtype, device="cuda"),
                                     torch.empty(max(E, 1), d_z, 0, dtype=dtype, device="cuda"), db=db)
        rows = [dZ[ptr[i]:ptr[i + 1]].double() for i in range(max(E, 1))]
        want, size = (torch.stack([r.sum(0) for r in x]) for x in (rows, [r.abs() for r in rows]))
        ref.check(db, want, ref.bound(want, size, T * k, dtype), "db")


# one turn of the largest tiles: whole ones, ragged ones, few steps
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("T,E,d_in,d_out", [(4096, 0, 512, 4096), (4000, 2, 520, 4072), (3900, 3, 72, 4088)])
def test_largest_tiles(gpu_lib, dtype, T, E, d_in, d_out):
    for act in ("none", "gelu"):
        Case(gpu_lib, T, 1, E, d_in, d_out, dtype, act).forward(bias=True, residual=act == "none", pre=True)
    Case(gpu_lib, T, 1, E, d_in, d_out // 2 // 8 * 8, dtype, "swiglu", dropped=0.1 if E else 0.0).forward(bias=True, residual=True, pre=True)
    c = Case(gpu_lib, T, 1, E, d_out, d_in, dtype, dropped=0.1 if E else 0.0)
    for act in ("none", "silu", "swiglu"):
        c.dx(act)


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("T,E,d_in,d_out", [(1024, 0, 4096, 4096), (1100, 1, 4072, 4088)])
def test_largest_tiles_of_weight_gradients(gpu_lib, dtype, T, E, d_in, d_out):
    c = Case(gpu_lib, T, 1, E, d_in, d_out, dtype)
    c.dw()
    c.dw(db=False)


@pytest.mark.parametrize("dtype", TYPES)
def test_many_experts(gpu_lib, dtype):
    """More experts than a wavefront has lanes, than LDS keeps by default, than there are rows."""
    for T, k, E, d in ((700, 2, 1000, 24), (3000, 8, 1024, 72), (5, 3, 700, 64)):
        c = Case(gpu_lib, T, k, E, d, 40, dtype, "silu", dropped=0.1)
        c.forward(bias=True, residual=False, pre=True)
        c.dx("gelu")
        c.dw()


@pytest.mark.parametrize("dtype", TYPES)
def test_experts_that_share_a_matrix(gpu_lib, dtype):
    """Weights and biases that are read may be one matrix for all experts."""
    for T in (3, 400):
        c = Case(gpu_lib, T, 2, 4, 64, 48, dtype, "gelu")
        W, bias = c.W[:1].expand(4, -1, -1), c.bias[:1].expand(4, -1)
        y = torch.empty(c.rows, 48, dtype=dtype, device="cuda")
        gpu_lib.sptir_moe_product(c.r, c.X_dev, c.W_dev[:1].expand(4, -1, -1), y, bias=c.bias_dev[:1].expand(4, -1), activation="gelu", gather=True)
        want, limit, _, _ = ref.product(c.parts, c.rows, c.X, W, bias, None, "gelu")
        ref.check(y, want, limit, "y")
        d = torch.empty(c.rows, 64, dtype=dtype, device="cuda")
        gpu_lib.sptir_moe_product_dx(c.r, c.dZ_dev, c.W_dev[:1].expand(4, -1, -1), d)
        want, limit = ref.product_dx(c.parts, c.rows, c.dZ, W, None, "none")
        ref.check(d, want, limit, "dX")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,k,E,width", [(40, 4, 12, 2048), (33, 9, 20, 2047), (20, 12, 16, 4100), (50, 3, 8, 2056), (2, 5, 9, 10000)])
def test_wide_rows(gpu_lib, dtype, T, k, E, width):
    """Rows that a whole workgroup takes, with choices on both sides of the gradient's rule."""
    say("wide rows", dtype, T, k, E, width)
    gen = torch.Generator().manual_seed(T + width)
    e = choices(gen, T, k, E, 0.2)
    ptr, entry, slot = ref.sort(e, E)
    kept, n = int(ptr[-1]), T * k
    r = gpu_lib.sptir_moe_sort(e.cuda(), E)
    X, Ys, dY = (randn(gen, rows, width, dtype=dtype) for rows in (T, n, T))
    Ys[kept:] = math.nan
    w = randn(gen, T, k)
    token = entry[:kept].long() // k
    xs, _ = out_like(n, width, dtype)
    gpu_lib.sptir_moe_gather(r, X.cuda(), xs)
    assert torch.equal(xs[:kept].cpu(), X[token]) and (xs[kept:] == 0).all()
    live = (slot.view(T, k) >= 0)[:, :, None]
    values = torch.where(live, Ys.double()[slot.long().clamp(min=0)].view(T, k, width), 0.0)
    terms = values * w.double()[:, :, None]
    y, _ = out_like(T, width, dtype)
    gpu_lib.sptir_moe_combine(r, Ys.cuda(), y, weights=w.cuda())
    ref.check(y, terms.sum(1), ref.bound(terms.sum(1), terms.abs().sum(1), k, dtype), "combine")
    d, _ = out_like(n, width, dtype)
    dw = torch.full((T, k), math.nan, device="cuda")
    gpu_lib.sptir_moe_combine_backward(r, dY.cuda(), Ys.cuda(), w.cuda(), d, dw)
    want = torch.zeros(n, width, dtype=torch.float64)
    want[:kept] = dY.double()[token] * w.double().view(-1)[entry[:kept].long()][:, None]
    ref.check(d, want, ref.bound(want, want.abs(), 1, dtype), "dYs")
    prod = dY.double()[:, None, :] * values
    ref.check(dw, prod.sum(2), ref.bound(prod.sum(2), prod.abs().sum(2), width, F32), "d_weights")


def test_sizes_of_the_workspace(gpu_lib):
    """None where a gradient is not split, the same for the same sizes, refused where it is too small or not there."""
    lib = moe._library()
    need = lib.sptir_moe_product_dw_workspace
    assert need(0, 1, 64, 64) == 0 and need(-1, 1, 64, 64) == 0 and need(100, 0, 64, 64) == 0 and need(1 << 20, 128, 4096, 4096) == 0
    for rows, E, d_in, d_z in ((10 ** 6, 1, 1, 1), (32768, 1, 1024, 2048), (2 ** 31 - 1, 4, 64, 64), (65536, 1, 0, 100)):
        size = need(rows, E, d_in, d_z)
        assert size > 0 and size == need(rows, E, d_in, d_z) and size <= 64 * 4 * E * d_z * (d_in + 8)
    dZ, X, dW = torch.ones(9000, 24, device="cuda"), torch.ones(9000, 40, device="cuda"), torch.full((24, 40), 7.0, device="cuda")
    q = moe._ProductDw(moe._PRODUCT_DW_SIZE, 0, 0, 0, 40, 24, 9000, dZ.data_ptr(), 24, X.data_ptr(), 40, dW.data_ptr(), 40, 0, None, 0, None, 0)
    size = need(9000, 1, 40, 24)
    ws = torch.empty(size + 16, dtype=torch.uint8, device="cuda")
    for at, given in ((None, size), (ws.data_ptr(), size - 1), (ws.data_ptr() + 4, size)):
        q.workspace, q.workspace_bytes = at, given
        assert lib.sptir_moe_product_dw(None, ctypes.byref(q), None) != 0
    torch.cuda.synchronize()
    assert (dW == 7).all()
