"""The experts' products of 8-bit integers against their definition in 64 bits: types, odd sizes, strides, dropped entries, empty experts,
the largest sums, scales that are not finite, streams and graphs."""
import math

import pytest
import torch

import moe8_reference as ref8
import moe_reference as ref
from test_gpu_moe import ACTS, BF16, F32, SHAPES, TYPES, choices, out_like, randn, say, strided

pytestmark = pytest.mark.gpu


def strided8(t, extra):
    if extra == 0:
        return t.cuda()
    wide = torch.full((*t.shape[:-1], t.shape[-1] + extra), 101, dtype=t.dtype, device="cuda")
    wide[..., :t.shape[-1]] = t.cuda()
    return wide[..., :t.shape[-1]]


class Case:
    def __init__(self, gpu_lib, T, k, E, d_in, d_out, dtype, act="none", dropped=0.0, gather=True, extra=0, skew=True):
        say("int8", T, k, E, d_in, d_out, dtype, act, dropped, gather, extra)
        self.lib, self.dtype, self.act, self.extra = gpu_lib, dtype, act, extra
        self.k, self.E, self.d_in, self.d_out, self.rows = k, max(E, 1), d_in, d_out, T * k
        self.wide = 2 * d_out if act == "swiglu" else d_out
        gen = torch.Generator().manual_seed(T + 7 * d_in + 13 * d_out)
        if E:
            e = choices(gen, T, k, E, dropped, skew)
            self.order, self.r = ref.sort(e, E), gpu_lib.sptir_moe_sort(e.cuda(), E)
            kept = int(self.order[0][-1])
        else:
            self.order, self.r, gather, kept = None, None, False, self.rows
        self.gather = gather
        self.parts = ref.groups(self.order, k, self.E, self.rows, gather)
        x_rows = T if gather else self.rows
        self.X = torch.randint(-128, 128, (x_rows, d_in), generator=gen, dtype=torch.int8)
        self.W = torch.randint(-128, 128, (self.E, self.wide, d_in), generator=gen, dtype=torch.int8)
        self.x_scales = torch.exp(randn(gen, x_rows)) / 128
        self.w_scales = torch.exp(randn(gen, self.E, self.wide)) / 128 * max(d_in, 1) ** -0.5
        self.bias, self.residual = randn(gen, self.E, self.wide, dtype=dtype), randn(gen, self.rows, d_out, dtype=dtype)
        if not gather:
            self.x_scales[kept:] = math.nan                # rows that belong to no expert reach nothing
        self.residual[kept:] = math.nan
        self.dev = {"X": strided8(self.X, extra), "W": strided8(self.W, extra), "residual": strided(self.residual, extra), "bias": self.bias.cuda(),
                    "x_scales": self.x_scales.cuda(), "w_scales": strided(self.w_scales, extra)}

    def call(self, y, bias=False, residual=False, pre=None, stream=None):
        d = self.dev
        self.lib.sptir_moe_product_int8(self.r, d["X"], d["x_scales"], d["W"], d["w_scales"], y, bias=d["bias"] if bias else None,
                                        residual=d["residual"] if residual else None, pre=pre, activation=self.act, gather=self.gather,
                                        stream=stream)

    def check(self, bias, residual, pre):
        y, rest = out_like(self.rows, self.d_out, self.dtype, self.extra)
        z, z_rest = out_like(self.rows, self.wide, self.dtype, self.extra)
        self.call(y, bias, residual, z if pre else None)
        want, limit, z_want, z_limit = ref8.product(self.parts, self.rows, self.X, self.x_scales, self.W, self.w_scales, self.bias if bias else None,
                                                    self.residual if residual else None, self.act, self.dtype)
        ref.check(y, want, limit, "y")
        assert torch.isnan(rest).all() and torch.isnan(z_rest).all()
        if pre:
            ref.check(z, z_want, z_limit, "pre")
        return y


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T,k,E,d_in,d_out", SHAPES)
def test_product(gpu_lib, dtype, act, T, k, E, d_in, d_out):
    c = Case(gpu_lib, T, k, E, d_in, d_out, dtype, act, dropped=0.15 if T > 3 and E else 0.0)
    c.check(bias=True, residual=True, pre=True)
    c.check(bias=False, residual=False, pre=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("extra", [1, 3, 8, 64])
def test_strides(gpu_lib, dtype, extra):
    """Rows that are not aligned to 16 bytes, X already in sorted order, other numbers between the rows."""
    for act, shape in (("swiglu", (70, 2, 4, 136, 80)), ("gelu", (300, 2, 3, 64, 200)), ("silu", (9, 2, 6, 72, 48)), ("none", (400, 2, 3, 128, 256))):
        Case(gpu_lib, *shape, dtype, act, dropped=0.1, gather=False, extra=extra).check(bias=True, residual=True, pre=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d_in,d_out", [(64, 64), (128, 256), (512, 96), (1024, 1024)])
@pytest.mark.parametrize("T,k,E", [(2000, 2, 8), (3000, 1, 0), (500, 4, 64)])
def test_whole_tiles(gpu_lib, dtype, d_in, d_out, T, k, E):
    Case(gpu_lib, T, k, E, d_in, d_out, dtype, "swiglu", skew=False).check(bias=True, residual=False, pre=True)


# (several wide tiles a workgroup, so that scales change places while an epilogue reads the last ones; by the choice's estimates)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act,T,k,E,d_in,d_out", [("swiglu", 8192, 2, 6, 256, 1024), ("gelu", 12000, 1, 0, 128, 2048), ("none", 9000, 2, 40, 192, 1536)])
def test_several_tiles_a_workgroup(gpu_lib, dtype, act, T, k, E, d_in, d_out):
    Case(gpu_lib, T, k, E, d_in, d_out, dtype, act, dropped=0.2 if E else 0.0).check(bias=True, residual=True, pre=False)


@pytest.mark.parametrize("T,k,E,dropped", [(60, 2, 3, 1.0), (1, 1, 9, 0.0), (400, 2, 5, 1.0)])
def test_experts_without_rows(gpu_lib, T, k, E, dropped):
    Case(gpu_lib, T, k, E, 64, 96, BF16, "silu", dropped=dropped).check(bias=True, residual=True, pre=True)


@pytest.mark.parametrize("rows", [3, 300])
def test_largest_sums(gpu_lib, rows):
    """131,071 products of (-128)^2 are below 2^31; one more product is refused."""
    d_in, wide = 131071, 48
    X, W = torch.full((rows, d_in), -128, dtype=torch.int8, device="cuda"), torch.full((wide, d_in), -128, dtype=torch.int8, device="cuda")
    W[1::2] = 127
    Y = torch.empty(rows, wide, device="cuda")
    gpu_lib.sptir_moe_product_int8(None, X, torch.full((rows,), 2.0 ** -20, device="cuda"), W, torch.ones(wide, device="cuda"), Y)
    want = torch.tensor([2.0 ** 14 * d_in, -127.0 * 128 * d_in]).repeat(wide // 2) * 2.0 ** -20
    assert float((Y.cpu() - want).abs().max()) <= 2.0 ** -24 * float(want.abs().max())
    more = torch.zeros(rows, d_in + 1, dtype=torch.int8, device="cuda")
    with pytest.raises(gpu_lib.SptirError) as caught:
        gpu_lib.sptir_moe_product_int8(None, more, torch.ones(rows, device="cuda"), more[:2], torch.ones(2, device="cuda"), Y[:, :2])
    assert caught.value.status == 6


@pytest.mark.parametrize("T", [5, 600])
def test_a_scale_that_is_no_number_reaches_its_row(gpu_lib, T):
    """A row that could not be quantised (scale NaN): its own rows of y are NaN, no others."""
    gen = torch.Generator().manual_seed(T)
    X = randn(gen, T, 128, dtype=BF16)
    X[3, 7] = math.inf
    X[1, 0] = math.nan
    Q, s = torch.empty(T, 128, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    gpu_lib.sptir_moe_quantise(X.cuda(), Q, s)
    W = torch.randint(-127, 128, (256, 128), generator=gen, dtype=torch.int8).cuda()
    Y = torch.empty(T, 256, dtype=BF16, device="cuda")
    gpu_lib.sptir_moe_product_int8(None, Q, s, W, torch.ones(256, device="cuda"), Y)
    bad = torch.isnan(Y).cpu()
    assert bad[[1, 3]].all()
    bad[[1, 3]] = False
    assert not bad.any()


def test_no_inputs(gpu_lib):
    """d_in 0: z is the bias."""
    for rows in (4, 500):
        X, W = torch.empty(rows, 0, dtype=torch.int8, device="cuda"), torch.empty(24, 0, dtype=torch.int8, device="cuda")
        bias = torch.arange(24, device="cuda").float()
        Y = torch.empty(rows, 24, device="cuda")
        gpu_lib.sptir_moe_product_int8(None, X, torch.zeros(rows, device="cuda"), W, torch.zeros(24, device="cuda"), Y, bias=bias)
        assert torch.equal(Y, bias.expand(rows, 24))


@pytest.mark.parametrize("rows", [6, 900])
def test_experts_that_share_weights(gpu_lib, rows):
    """W and its scales of stride 0: one matrix for all experts."""
    gen = torch.Generator().manual_seed(rows)
    e = torch.randint(0, 5, (rows, 1), generator=gen, dtype=torch.int32)
    r = gpu_lib.sptir_moe_sort(e.cuda(), 5)
    X = torch.randint(-127, 128, (rows, 96), generator=gen, dtype=torch.int8)
    W, ws, xs = torch.randint(-127, 128, (1, 40, 96), generator=gen, dtype=torch.int8), torch.rand(1, 40, generator=gen), torch.rand(rows, generator=gen)
    Y = torch.empty(rows, 40, device="cuda")
    gpu_lib.sptir_moe_product_int8(r, X.cuda(), xs.cuda(), W.cuda().expand(5, 40, 96), ws.cuda().expand(5, 40), Y, gather=True)
    at = r.entry_of.cpu().long()
    want = (X[at].double() @ W[0].double().t()) * xs[at].double()[:, None] * ws[0].double()
    ref.check(Y, want, want.abs() * 2.0 ** -22 + 2.0 ** -126, "y")


def test_in_a_graph_and_on_streams(gpu_lib):
    """Quantise and product, captured together and replayed with new inputs, and on another stream, give the bits of eager calls."""
    T, k, E, K, N = 300, 2, 6, 256, 192
    gen = torch.Generator().manual_seed(0)
    c = Case(gpu_lib, T, k, E, K, N, BF16, "swiglu")
    inputs = [randn(gen, T, K, dtype=BF16).cuda() for _ in range(3)]
    X, Y = inputs[0].clone(), torch.empty(T * k, N, dtype=BF16, device="cuda")

    def step(stream=None):
        gpu_lib.sptir_moe_quantise(X, c.dev["X"], c.dev["x_scales"], stream=stream)
        c.call(Y, bias=True, stream=stream)

    want = []
    for x in inputs:
        X.copy_(x)
        step()
        want.append(Y.clone())
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step()
    for n in range(6):
        X.copy_(inputs[n % 3])
        Y.fill_(math.nan)
        graph.replay()
        assert torch.equal(Y, want[n % 3])
        inputs[0].float().sum().item()
    torch.cuda.synchronize()
    for n in range(6):
        X.copy_(inputs[n % 3])
        Y.fill_(math.nan)
        side.wait_stream(torch.cuda.current_stream())
        step(side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(Y, want[n % 3])


def test_refusals(gpu_lib):
    X, W = torch.zeros(4, 32, dtype=torch.int8, device="cuda"), torch.zeros(2, 16, 32, dtype=torch.int8, device="cuda")
    xs, ws, Y = torch.zeros(4, device="cuda"), torch.zeros(2, 16, device="cuda"), torch.zeros(4, 16, device="cuda")
    r = gpu_lib.sptir_moe_sort(torch.zeros(4, 1, dtype=torch.int32, device="cuda"), 2)
    call = gpu_lib.sptir_moe_product_int8
    call(r, X, xs, W, ws, Y)
    for args in ((r, X, xs[:3], W, ws, Y), (r, X[:3], xs, W, ws, Y), (r, X, xs, W[:1], ws, Y), (r, X, xs, W, ws[:, :15], Y), (r, X, xs, W, ws, Y[:, :15]),
                 (None, X, xs, W, ws, Y)):
        with pytest.raises(ValueError):
            call(*args)
    for args in ((r, X.float(), xs, W, ws, Y), (r, X, xs.double(), W, ws, Y), (r, X, xs, W.float(), ws, Y), (r, X, xs, W, ws.half(), Y),
                 (r, X, xs, W, ws, Y.to(torch.int8)), (r, X, None, W, ws, Y)):
        with pytest.raises(TypeError):
            call(*args)
    with pytest.raises(ValueError):
        call(r, X, xs, W, ws, Y, activation="exp")
    with pytest.raises(gpu_lib.SptirError):
        call(r, X, xs, W, ws, Y, pre=Y)
