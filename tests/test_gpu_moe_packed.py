"""Gradients that read activations kept in 8 bits: dX through the derivative at a kept z, dW with a kept x; against the definition on what
is kept, and bit for bit against the gradients that read the same values in their type."""
import math

import pytest
import torch

import moe8_reference as ref8
import moe_reference as ref
from test_gpu_moe import BF16, F16, F32, SHAPES, TYPES, Case, out_like, randn, say, strided
from test_gpu_moe_int8 import strided8
from test_gpu_moe_rows8 import packed

pytestmark = pytest.mark.gpu
ACTS = ["relu", "gelu", "silu", "swiglu"]


def kept_of(lib, X, extra):
    """(codes and exponents on the GPU, what they stand for)"""
    Q, E = packed(lib, torch.nan_to_num(X), 0)
    Q, E = strided8(Q.cpu(), extra), strided8(E.cpu(), extra)
    return Q, E, ref8.kept(Q.cpu(), E.cpu(), X.dtype)


def check_dx(c, act):
    wide = 2 * c.d_in if act == "swiglu" else c.d_in
    pre = randn(c.gen, c.rows, wide, dtype=c.dtype, scale=2.0)
    Q, E, values = kept_of(c.lib, pre, c.extra)
    d, rest = out_like(c.rows, wide, c.dtype, c.extra)
    c.lib.sptir_moe_product_dx_packed(c.r, c.dZ_dev, c.W_dev, d, Q, E, activation=act)
    want, limit = ref.product_dx(c.parts, c.rows, c.dZ, c.W, values, act)
    ref.check(d, want, limit, "dX " + act)
    assert torch.isnan(rest).all()
    plain, _ = out_like(c.rows, wide, c.dtype, c.extra)
    c.lib.sptir_moe_product_dx(c.r, c.dZ_dev, c.W_dev, plain, pre=strided(values, c.extra), activation=act)
    if c.extra % 8 == 0:  # (the same kernel: the same bits)
        assert torch.equal(torch.nan_to_num(d), torch.nan_to_num(plain))


def check_dw(c, db=True):
    Q, E, values = kept_of(c.lib, c.X, c.extra)
    if not c.gather and c.order is not None:
        E[int(c.order[0][-1]):] = 255                      # rows that belong to no expert reach nothing
    dW = strided(torch.full((c.E, c.wide, c.d_in), math.nan, dtype=c.dtype), c.extra)
    b = torch.full((c.E, c.wide), math.nan, dtype=c.dtype, device="cuda") if db else None
    c.lib.sptir_moe_product_dw_packed(c.r, c.dZ_dev, Q, E, dW, db=b, gather=c.gather)
    want, limit, b_want, b_limit = ref.product_dw(c.parts, c.dZ, values, c.E)
    ref.check(dW, want, limit, "dW")
    if db:
        ref.check(b, b_want, b_limit, "db")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,k,E,d_in,d_out", SHAPES)
def test_gradients(gpu_lib, dtype, T, k, E, d_in, d_out):
    c = Case(gpu_lib, T, k, E, d_in, d_out, dtype, "none", dropped=0.15 if T > 3 and E else 0.0, seed=5)
    for act in ACTS:
        check_dx(c, act)
    check_dw(c)
    check_dw(c, db=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("extra", [1, 3, 8, 64])
def test_strides(gpu_lib, dtype, extra):
    for act, shape in (("swiglu", (70, 2, 4, 136, 80)), ("gelu", (300, 2, 3, 64, 200)), ("silu", (9, 2, 6, 72, 48)), ("swiglu", (40, 2, 3, 76, 32))):
        c = Case(gpu_lib, *shape, dtype, "none", dropped=0.1, gather=False, extra=extra)
        check_dx(c, act)
        check_dw(c)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d_in,d_out", [(64, 64), (128, 256), (1024, 1024)])
@pytest.mark.parametrize("T,k,E", [(2000, 2, 8), (3000, 1, 0), (500, 4, 64)])
def test_whole_tiles(gpu_lib, dtype, d_in, d_out, T, k, E):
    c = Case(gpu_lib, T, k, E, d_in, d_out, dtype, "none", skew=False)
    check_dx(c, "swiglu")
    check_dx(c, "gelu")
    check_dw(c)


def test_many_rows_and_few_weights(gpu_lib):
    """Rows in parts, joined: the gradient's own workspace and that of x in one."""
    from paper_2207_04606_amd import moe
    lib = moe._library()
    assert lib.sptir_moe_product_dw_workspace(9000, 1, 40, 24) > 0
    assert lib.sptir_moe_product_dw_packed_workspace(2, 9000, 9000, 1, 40, 24) >= lib.sptir_moe_product_dw_workspace(9000, 1, 40, 24) + 9000 * 80
    for dtype in TYPES:
        check_dw(Case(gpu_lib, 9000, 1, 0, 40, 24, dtype, "none"))
        check_dw(Case(gpu_lib, 6000, 2, 3, 41, 24, dtype, "none", dropped=0.1))


def test_a_block_that_is_no_number_reaches_what_reads_it(gpu_lib):
    """An infinity in x: the columns of its block of that expert's dW, and no others."""
    gen = torch.Generator().manual_seed(2)
    T, E, K, N = 200, 3, 96, 64
    e = torch.randint(0, E, (T, 1), generator=gen, dtype=torch.int32)
    r = gpu_lib.sptir_moe_sort(e.cuda(), E)
    X, dZ = randn(gen, T, K, dtype=BF16), randn(gen, T, N, dtype=BF16)
    X[17, 40] = math.inf
    Q, X_e = packed(gpu_lib, X)
    dW = torch.empty(E, N, K, dtype=BF16, device="cuda")
    gpu_lib.sptir_moe_product_dw_packed(r, dZ.cuda(), Q, X_e, dW, gather=True)
    bad = torch.isnan(dW).cpu()
    assert bad[int(e[17, 0]), :, 32:64].all()
    bad[int(e[17, 0]), :, 32:64] = False
    assert not bad.any()


@pytest.mark.parametrize("act", ACTS)
def test_gradient_against_differences(gpu_lib, act):
    """float32: a step of the kept z along a direction changes <dZ W, act(z)> as dX says."""
    gen = torch.Generator().manual_seed(9)
    rows, d_in, d_z, step = 30, 64, 48, 2.0 ** -5
    wide = 2 * d_in if act == "swiglu" else d_in
    z = randn(gen, rows, wide).round() / 2 + 0.25          # (no step crosses the corner of relu)
    dZ, W = randn(gen, rows, d_z), randn(gen, d_z, d_in)
    Q, E = packed(gpu_lib, z)
    kept = ref8.kept(Q.cpu(), E.cpu(), F32)
    assert torch.equal(kept, z)                            # (multiples of a quarter below 8)
    d = torch.empty(rows, wide, device="cuda")
    gpu_lib.sptir_moe_product_dx_packed(None, dZ.cuda(), W.cuda(), d, Q, E, activation=act)
    direction = torch.sign(randn(gen, rows, wide)).double()
    of = dZ.double() @ W.double()
    slope = (of * (ref.activation(z.double() + step * direction, act) - ref.activation(z.double() - step * direction, act))).sum(1) / (2 * step)
    want = (d.cpu().double() * direction).sum(1)
    # third derivatives of the activations are below 3 (of swiglu's along a sign vector 3 (1 + |u|)); sums in float32
    third = 3.0 * (1.0 + z.abs().max()) if act == "swiglu" else 3.0
    limit = of.abs().sum(1) * third * step ** 2 / 6 + 2.0 ** -17 * of.abs().sum(1) * (1.0 + float(z.abs().max()))
    assert ((slope - want).abs() <= limit).all()


def test_in_a_graph(gpu_lib):
    """Packed in the forward pass, read in the backward pass, captured together: replays with new inputs give the bits of eager calls."""
    gen = torch.Generator().manual_seed(4)
    T, k, E, D, H = 500, 2, 5, 128, 96
    e = torch.randint(0, E, (T, k), generator=gen, dtype=torch.int32)
    r = gpu_lib.sptir_moe_sort(e.cuda(), E)
    inputs = [(randn(gen, T, D, dtype=BF16).cuda(), randn(gen, T * k, 2 * H, dtype=BF16).cuda()) for _ in range(3)]
    d_ys, W2 = randn(gen, T * k, D, dtype=BF16).cuda(), randn(gen, E, D, H, dtype=BF16).cuda()
    X, pre = inputs[0][0].clone(), inputs[0][1].clone()
    Q, X_e = torch.empty(T, D, dtype=torch.int8, device="cuda"), torch.empty(T, D // 32, dtype=torch.uint8, device="cuda")
    P, P_e = torch.empty(T * k, 2 * H, dtype=torch.int8, device="cuda"), torch.empty(T * k, 2 * H // 32, dtype=torch.uint8, device="cuda")
    d_pre, h = torch.empty_like(pre), torch.empty(T * k, H, dtype=BF16, device="cuda")
    dW1, dW2 = torch.empty(E, 2 * H, D, dtype=BF16, device="cuda"), torch.empty_like(W2)

    def step(stream=None):
        gpu_lib.sptir_moe_pack(X, Q, X_e, stream=stream)
        gpu_lib.sptir_moe_pack(pre, P, P_e, stream=stream)
        gpu_lib.sptir_moe_product_dx_packed(r, d_ys, W2, d_pre, P, P_e, activation="swiglu", stream=stream)
        gpu_lib.sptir_moe_product_dw_packed(r, d_pre, Q, X_e, dW1, gather=True, stream=stream)
        gpu_lib.sptir_moe_unpack(P, P_e, h, activation="swiglu", stream=stream)
        gpu_lib.sptir_moe_product_dw(r, d_ys, h, dW2, stream=stream)

    def outputs():
        return d_pre, h, dW1, dW2

    want = []
    for x, z in inputs:
        X.copy_(x)
        pre.copy_(z)
        step()
        want.append([t.clone() for t in outputs()])
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step()
    for n in range(6):
        X.copy_(inputs[n % 3][0])
        pre.copy_(inputs[n % 3][1])
        for t in outputs():
            t.fill_(math.nan)
        graph.replay()
        assert all(torch.equal(t, w) for t, w in zip(outputs(), want[n % 3]))
        inputs[0][0].float().sum().item()
        step()
        assert all(torch.equal(t, w) for t, w in zip(outputs(), want[n % 3]))
    side.wait_stream(torch.cuda.current_stream())
    for t in outputs():
        t.fill_(math.nan)
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(t, w) for t, w in zip(outputs(), want[2]))


def test_refusals(gpu_lib):
    dZ, W, dX = torch.zeros(4, 16, device="cuda"), torch.zeros(16, 64, device="cuda"), torch.zeros(4, 64, device="cuda")
    Q, E = torch.zeros(4, 64, dtype=torch.int8, device="cuda"), torch.zeros(4, 2, dtype=torch.uint8, device="cuda")
    gpu_lib.sptir_moe_product_dx_packed(None, dZ, W, dX, Q, E, activation="relu")
    for args, act in (((None, dZ, W, dX, Q, E), "none"), ((None, dZ, W, dX, Q, E), "exp"), ((None, dZ, W, dX, Q[:, :63], E), "relu"),
                      ((None, dZ, W, dX, Q, E[:, :1]), "relu"), ((None, dZ, W, dX, Q, E), "swiglu")):
        with pytest.raises(ValueError):
            gpu_lib.sptir_moe_product_dx_packed(*args, activation=act)
    with pytest.raises(TypeError):
        gpu_lib.sptir_moe_product_dx_packed(None, dZ, W, dX, Q.float(), E, activation="relu")
    dW = torch.zeros(16, 64, device="cuda")
    gpu_lib.sptir_moe_product_dw_packed(None, dZ, Q, E, dW)
    for args in ((None, dZ, Q[:3], E[:3], dW), (None, dZ, Q, E[:, :1], dW), (None, dZ, Q, E, dW[:, :63])):
        with pytest.raises(ValueError):
            gpu_lib.sptir_moe_product_dw_packed(*args)
    with pytest.raises(TypeError):
        gpu_lib.sptir_moe_product_dw_packed(None, dZ, Q, E.to(torch.int8), dW)
