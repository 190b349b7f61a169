"""The operators of a mixture-of-experts layer against their definitions in 64 bits (tests/moe_reference.py), through the
public entry points: types, odd sizes, strides, dropped entries, masked logits, empty experts, refusals."""
import math

import pytest
import torch

import moe_reference as ref

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]


def say(*what):
    print("[moe]", *what, flush=True)


def randn(gen, *shape, dtype=F32, scale=1.0):
    return (torch.randn(*shape, generator=gen) * scale).to(dtype)


def strided(t, extra):
    """The same matrix on the GPU inside a wider one whose other columns are NaN."""
    if extra == 0:
        return t.cuda()
    wide = torch.full((*t.shape[:-1], t.shape[-1] + extra), math.nan, dtype=t.dtype, device="cuda")
    wide[..., :t.shape[-1]] = t.cuda()
    return wide[..., :t.shape[-1]]


def out_like(rows, cols, dtype, extra=0):
    """(output, the columns behind it, which nothing may write)"""
    whole = torch.full((rows, cols + extra), math.nan, dtype=dtype, device="cuda")
    return whole[:, :cols], whole[:, cols:]


def choices(gen, T, k, E, dropped=0.0, skew=True):
    """Distinct experts of every token, some of them -1; the second half of the experts rarely chosen."""
    score = torch.randn(T, E, generator=gen) + (torch.arange(E) < (E + 1) // 2) * (2.0 if skew else 0.0)
    e = torch.argsort(score, dim=1, descending=True)[:, :k].to(torch.int32).contiguous()
    if dropped:
        e[torch.rand(T, k, generator=gen) < dropped] = -1
    return e


# ------------------------------------------------------------------------------------------------ router
def masked_logits(gen, T, E, dtype):
    l = randn(gen, T, E, scale=2.0).to(dtype)
    l[::7] = (l[::7] * 2).round() / 2                      # many ties
    if T > 3:
        l[1] = -math.inf                                   # no expert left
        l[2] = torch.finfo(dtype).min                      # the type's lowest value is still a logit
        l[3, 1:] = -math.inf                               # one left
    if T > 20:
        l[10:20][torch.rand(10, E, generator=gen) < 0.5] = -math.inf
    return l


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("normalise", [True, False])
@pytest.mark.parametrize("T,E,k,extra", [(1, 1, 1, 0), (1, 64, 8, 0), (5, 3, 2, 5), (37, 8, 2, 0), (70, 60, 6, 4), (129, 65, 64, 1),
                                         (64, 128, 8, 0), (33, 200, 7, 3), (300, 16, 4, 0), (9, 1000, 16, 0), (6, 1024, 1, 8)])
def test_route(gpu_lib, dtype, normalise, T, E, k, extra):
    say("route", dtype, normalise, T, E, k)
    gen = torch.Generator().manual_seed(T * 1000 + E + k)
    l = masked_logits(gen, T, E, dtype)
    want, w_want = ref.route(l, k, normalise)
    dev = strided(l, extra)
    experts = torch.full((T, k), -7, dtype=torch.int32, device="cuda")
    weights = torch.full((T, k), math.nan, device="cuda")
    gpu_lib.sptir_moe_route(dev, experts, weights, normalise=normalise)
    assert torch.equal(experts.cpu(), want)
    # exp of a float32 difference below 180 (that is 2^-24 * 180 relative), its own rounding, a sum of positive terms
    logits_range = 2.0 ** -24 * 200.0
    ref.check(weights, w_want, w_want * (logits_range + (math.sqrt(E) + 8) * 2.0 ** -22) + 1e-37, "weights")
    dw = randn(gen, T, k)
    dw[want < 0] = math.nan                                # of a choice that is none
    want_d = ref.route_gradient(l, want, dw, normalise)
    d, rest = out_like(T, E, dtype, extra)
    gpu_lib.sptir_moe_route_backward(dev, experts, weights, dw.cuda(), d, normalise=normalise)
    size = float(torch.where(want < 0, torch.zeros_like(dw), dw).abs().max()) * 2
    limit = 1.01 * ref.UNIT[dtype] * want_d.abs() + size * (logits_range + (math.sqrt(E) + k + 16) * 2.0 ** -22) + ref.TINY[dtype]
    ref.check(d, want_d, limit, "d_logits")
    assert torch.isnan(rest).all()


def test_route_nan_and_infinity(gpu_lib):
    """A NaN that the sum runs over shows in the weights of its token only, and is never chosen."""
    l = torch.zeros(4, 8)
    l[1, 3] = math.nan
    l[2, 5] = math.inf
    for normalise in (True, False):
        experts = torch.empty(4, 2, dtype=torch.int32, device="cuda")
        weights = torch.empty(4, 2, device="cuda")
        gpu_lib.sptir_moe_route(l.cuda(), experts, weights, normalise=normalise)
        w = weights.cpu()
        assert experts.cpu().tolist() == [[0, 1], [0, 1], [5, 0], [0, 1]]
        assert torch.isnan(w[2, 0]) and torch.isfinite(w[0]).all() and torch.isfinite(w[3]).all()
        assert torch.isnan(w[1]).all() == (not normalise)


@pytest.mark.parametrize("normalise", [True, False])
def test_route_gradient_against_differences(gpu_lib, normalise):
    T, E, k, step = 40, 24, 3, 2.0 ** -6
    gen = torch.Generator().manual_seed(3)
    # logits of a token at least 3 steps apart, so that a step changes no choice
    l = torch.stack([torch.randperm(E, generator=gen) for _ in range(T)]).float() * 0.125
    dw, direction = randn(gen, T, k).cuda(), torch.sign(randn(gen, T, E)).cuda()
    l = l.cuda()

    def forward(at):
        experts = torch.empty(T, k, dtype=torch.int32, device="cuda")
        weights = torch.empty(T, k, device="cuda")
        gpu_lib.sptir_moe_route(at, experts, weights, normalise=normalise)
        return experts, weights

    experts, weights = forward(l)
    d = torch.empty_like(l)
    gpu_lib.sptir_moe_route_backward(l, experts, weights, dw, d, normalise=normalise)
    (e0, w0), (e1, w1) = forward(l - step * direction), forward(l + step * direction)
    assert torch.equal(e0, experts) and torch.equal(e1, experts)
    slope = ((w1.double() - w0.double()) * dw.double()).sum(1) / (2 * step)
    want = (d.double() * direction.double()).sum(1)
    # third derivative of a softmax entry along a sign vector: below 8; two float32 weights over the step
    limit = dw.double().abs().sum(1) * (8 * step ** 2 / 6 + 2.0 ** -22 / step)
    assert ((slope - want).abs() <= limit).all()


# ------------------------------------------------------------------------------------------------ sort
@pytest.mark.parametrize("T,k,E", [(0, 2, 4), (1, 1, 1), (1, 8, 64), (7, 3, 5), (100, 2, 1024), (1000, 6, 60), (16384, 1, 7), (16385, 1, 7),
                                   (4097, 4, 128), (40000, 8, 33), (3001, 7, 1000)])
@pytest.mark.parametrize("kind", ["random", "dropped", "one", "none"])
def test_sort(gpu_lib, T, k, E, kind):
    say("sort", T, k, E, kind)
    gen = torch.Generator().manual_seed(T + k + E)
    e = torch.randint(0, E, (T, k), generator=gen, dtype=torch.int32)
    if kind == "dropped":  # ids of other machines' experts, on both sides
        e = torch.randint(-E, 2 * E, (T, k), generator=gen, dtype=torch.int32)
    elif kind == "one":
        e[:] = E - 1
    elif kind == "none":
        e[:] = torch.tensor([-1, E, 2 ** 31 - 1, -2 ** 31])[torch.arange(T * k) % 4].view(T, k).to(torch.int32)
    r = gpu_lib.sptir_moe_sort(e.cuda(), E)
    for got, want, name in zip((r.expert_ptr, r.entry_of, r.slot_of), ref.sort(e, E), ("expert_ptr", "entry_of", "slot_of")):
        assert torch.equal(got.cpu(), want), name
    again = gpu_lib.sptir_moe_sort(e.cuda().flip(0).contiguous(), E, routing=r)  # into the arrays that are there
    assert again is r
    for got, want in zip((r.expert_ptr, r.entry_of, r.slot_of), ref.sort(e.flip(0), E)):
        assert torch.equal(got.cpu(), want)


# ------------------------------------------------------------------------------------------------ rows
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,k,E,width,extra,dropped", [(1, 1, 1, 1, 0, 0.0), (1, 8, 64, 256, 0, 0.0), (5, 2, 3, 7, 2, 0.3), (40, 3, 12, 111, 0, 0.2),
                                                       (33, 2, 4, 520, 8, 0.1), (64, 4, 8, 1024, 0, 1.0), (100, 1, 6, 2056, 0, 0.0),
                                                       (17, 6, 16, 4099, 5, 0.2), (300, 2, 8, 64, 64, 0.0), (9, 64, 70, 72, 0, 0.1)])
def test_rows(gpu_lib, dtype, T, k, E, width, extra, dropped):
    say("rows", dtype, T, k, E, width, extra, dropped)
    gen = torch.Generator().manual_seed(T + width)
    e = choices(gen, T, k, E, dropped)
    ptr, entry, slot = ref.sort(e, E)
    kept = int(ptr[-1])
    n = T * k
    r = gpu_lib.sptir_moe_sort(e.cuda(), E)
    X, Ys, dY, R = (randn(gen, rows, width, dtype=dtype) for rows in (T, n, T, T))
    Ys[kept:] = math.nan                                   # rows that belong to no entry are not read
    w = randn(gen, T, k)
    w[e < 0] = math.nan
    live = slot.view(T, k) >= 0
    s_of, token = slot.long().clamp(min=0), entry[:kept].long() // k
    dev = {name: strided(t, extra) for name, t in (("X", X), ("Ys", Ys), ("dY", dY), ("R", R))}

    def sorted_rows(values):
        out = torch.zeros(n, width, dtype=torch.float64)
        out[:kept] = values
        return out

    # gather, without and with weights
    for weights in (None, w):
        o, rest = out_like(n, width, dtype, extra)
        gpu_lib.sptir_moe_gather(r, dev["X"], o, weights=None if weights is None else w.cuda())
        want = X.double()[token]
        if weights is not None:
            want = want * w.double().view(-1)[entry[:kept].long()][:, None]
        want = sorted_rows(want)
        ref.check(o, want, ref.bound(want, want.abs(), 1, dtype) * (0.0 if weights is None else 1.0), "gather")
        assert torch.isnan(rest).all()
    # combine
    terms = torch.where(live[:, :, None], torch.where(live, w, 0.0).double()[:, :, None] * torch.nan_to_num(Ys.double())[s_of].view(T, k, width), 0.0)
    plain = torch.where(live[:, :, None], torch.nan_to_num(Ys.double())[s_of].view(T, k, width), 0.0)
    for weights, residual, parts in ((w, R, terms), (w, None, terms), (None, R, plain), (None, None, plain)):
        o, rest = out_like(T, width, dtype, extra)
        base = torch.zeros(T, width, dtype=torch.float64) if residual is None else R.double()
        want = parts.sum(1) + base
        gpu_lib.sptir_moe_combine(r, dev["Ys"], o, weights=None if weights is None else w.cuda(),
                                  residual=None if residual is None else dev["R"])
        ref.check(o, want, ref.bound(want, parts.abs().sum(1) + base.abs(), k + 1, dtype), "combine")
        assert torch.isnan(rest).all()
    in_place = strided(R, extra)
    gpu_lib.sptir_moe_combine(r, dev["Ys"], in_place, weights=w.cuda(), residual=in_place)
    want = terms.sum(1) + R.double()
    ref.check(in_place, want, ref.bound(want, terms.abs().sum(1) + R.double().abs(), k + 1, dtype), "combine in place")
    # gradients
    for weights, wanted in ((w, True), (None, True), (w, False)):
        o, rest = out_like(n, width, dtype, extra)
        dw = torch.full((T, k), math.nan, device="cuda") if wanted else None
        gpu_lib.sptir_moe_combine_backward(r, dev["dY"], dev["Ys"] if wanted else None, None if weights is None else w.cuda(), o, dw)
        want = dY.double()[token]
        if weights is not None:
            want = want * w.double().view(-1)[entry[:kept].long()][:, None]
        want = sorted_rows(want)
        ref.check(o, want, ref.bound(want, want.abs(), 1, dtype), "dYs")
        assert torch.isnan(rest).all()
        if wanted:
            prod = dY.double()[:, None, :] * plain
            ref.check(dw, prod.sum(2), ref.bound(prod.sum(2), prod.abs().sum(2), width, F32), "d_weights")


def test_combine_gradient_against_differences(gpu_lib):
    """The sum is linear in Ys and in the weights: one step of any size gives the slope up to rounding."""
    T, k, E, width = 50, 3, 7, 96
    gen = torch.Generator().manual_seed(1)
    r = gpu_lib.sptir_moe_sort(choices(gen, T, k, E, 0.1).cuda(), E)
    Ys, step, dY = (randn(gen, rows, width).cuda() for rows in (T * k, T * k, T))
    w, w_step = randn(gen, T, k).cuda(), randn(gen, T, k).cuda()

    def loss(ys, weights):
        y = torch.empty(T, width, device="cuda")
        gpu_lib.sptir_moe_combine(r, ys, y, weights=weights)
        return float((y.double() * dY.double()).sum())

    dYs, dw = torch.empty_like(Ys), torch.empty_like(w)
    gpu_lib.sptir_moe_combine_backward(r, dY, Ys, w, dYs, dw)
    size = float((dYs.double() * Ys.double()).abs().sum() + (dYs.double() * step.double()).abs().sum() + (dw.double() * w_step.double()).abs().sum())
    for got, want in ((loss(Ys + step, w) - loss(Ys, w), float((dYs.double() * step.double()).sum())),
                      (loss(Ys, w + w_step) - loss(Ys, w), float((dw.double() * w_step.double()).sum()))):
        assert abs(got - want) <= 2.0 ** -20 * size


# ------------------------------------------------------------------------------------------------ products
ACTS = ["none", "relu", "gelu", "silu", "swiglu"]


class Case:
    def __init__(self, gpu_lib, T, k, E, d_in, d_out, dtype, act="none", dropped=0.0, gather=True, extra=0, seed=0, skew=True):
        say("product", T, k, E, d_in, d_out, dtype, act, dropped, gather, extra)
        self.lib, self.dtype, self.act, self.extra = gpu_lib, dtype, act, extra
        self.k, self.E, self.d_in, self.d_out = k, max(E, 1), d_in, d_out
        self.wide = 2 * d_out if act == "swiglu" else d_out
        self.rows = T * k
        gen = self.gen = torch.Generator().manual_seed(seed + T + 7 * d_in + 13 * d_out)
        if E:
            e = choices(gen, T, k, E, dropped, skew)
            self.order, self.r = ref.sort(e, E), gpu_lib.sptir_moe_sort(e.cuda(), E)
            kept = int(self.order[0][-1])
        else:
            self.order, self.r, gather, kept = None, None, False, self.rows
        self.gather = gather
        self.parts = ref.groups(self.order, k, self.E, self.rows, gather)
        self.X = randn(gen, T if gather else self.rows, d_in, dtype=dtype)
        self.W = randn(gen, self.E, self.wide, d_in, dtype=dtype, scale=max(d_in, 1) ** -0.5)
        self.bias = randn(gen, self.E, self.wide, dtype=dtype)
        self.residual = randn(gen, self.rows, d_out, dtype=dtype)
        self.dZ = randn(gen, self.rows, self.wide, dtype=dtype)
        if not gather:
            self.X[kept:] = math.nan                        # rows that belong to no expert are not read
        self.dZ[kept:] = math.nan
        self.residual[kept:] = math.nan
        for name in ("X", "W", "residual", "dZ"):
            setattr(self, name + "_dev", strided(getattr(self, name), extra))
        self.bias_dev = self.bias.cuda()

    def forward(self, bias, residual, pre):
        y, rest = out_like(self.rows, self.d_out, self.dtype, self.extra)
        z, z_rest = out_like(self.rows, self.wide, self.dtype, self.extra)
        self.lib.sptir_moe_product(self.r, self.X_dev, self.W_dev, y, bias=self.bias_dev if bias else None,
                                   residual=self.residual_dev if residual else None, pre=z if pre else None,
                                   activation=self.act, gather=self.gather)
        want, limit, z_want, z_limit = ref.product(self.parts, self.rows, self.X, self.W, self.bias if bias else None,
                                                   self.residual if residual else None, self.act)
        ref.check(y, want, limit, "y")
        assert torch.isnan(rest).all() and torch.isnan(z_rest).all()
        if pre:
            ref.check(z, z_want, z_limit, "pre")

    def dx(self, act):
        wide = 2 * self.d_in if act == "swiglu" else self.d_in
        pre = randn(self.gen, self.rows, wide, dtype=self.dtype, scale=2.0)
        d, rest = out_like(self.rows, wide, self.dtype, self.extra)
        self.lib.sptir_moe_product_dx(self.r, self.dZ_dev, self.W_dev, d, pre=strided(pre, self.extra), activation=act)
        want, limit = ref.product_dx(self.parts, self.rows, self.dZ, self.W, pre, act)
        ref.check(d, want, limit, "dX " + act)
        assert torch.isnan(rest).all()

    def dw(self, db=True):
        dW = strided(torch.full((self.E, self.wide, self.d_in), math.nan, dtype=self.dtype), self.extra)
        b = torch.full((self.E, self.wide), math.nan, dtype=self.dtype, device="cuda") if db else None
        self.lib.sptir_moe_product_dw(self.r, self.dZ_dev, self.X_dev, dW, db=b, gather=self.gather)
        want, limit, b_want, b_limit = ref.product_dw(self.parts, self.dZ, self.X, self.E)
        ref.check(dW, want, limit, "dW")
        if db:
            ref.check(b, b_want, b_limit, "db")


# one token; few rows an expert; ragged tiles; more than a tile of every kind; odd sizes; one group; one expert of many
SHAPES = [(1, 8, 64, 256, 128), (1, 1, 1, 1, 1), (3, 2, 5, 7, 9), (12, 4, 8, 96, 160), (40, 3, 6, 200, 72), (130, 2, 3, 64, 300),
          (700, 2, 4, 128, 264), (257, 1, 0, 328, 136), (600, 2, 12, 72, 64), (1100, 1, 1, 136, 520), (64, 1, 0, 1000, 777),
          (33, 2, 4, 2048, 40)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T,k,E,d_in,d_out", SHAPES)
def test_product(gpu_lib, dtype, act, T, k, E, d_in, d_out):
    c = Case(gpu_lib, T, k, E, d_in, d_out, dtype, act, dropped=0.15 if T > 3 and E else 0.0)
    c.forward(bias=True, residual=True, pre=True)
    c.forward(bias=False, residual=False, pre=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,k,E,d_in,d_out", SHAPES)
def test_product_gradients(gpu_lib, dtype, T, k, E, d_in, d_out):
    c = Case(gpu_lib, T, k, E, d_in, d_out, dtype, "none", dropped=0.15 if T > 3 and E else 0.0, seed=5)
    for act in ACTS:
        c.dx(act)
    c.dw()
    c.dw(db=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("extra", [1, 3, 8, 64])
def test_product_strides(gpu_lib, dtype, extra):
    """Rows that are not aligned to 16 bytes, X already in sorted order, NaN between the rows."""
    for act, shape in (("swiglu", (70, 2, 4, 136, 80)), ("gelu", (300, 2, 3, 64, 200)), ("silu", (9, 2, 6, 72, 48))):
        c = Case(gpu_lib, *shape, dtype, act, dropped=0.1, gather=False, extra=extra)
        c.forward(bias=True, residual=True, pre=True)
        c.dx(act)
        c.dw()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d_in,d_out", [(64, 64), (128, 256), (512, 96), (1024, 1024)])
@pytest.mark.parametrize("T,k,E", [(2000, 2, 8), (3000, 1, 0), (500, 4, 64)])
def test_product_of_whole_tiles(gpu_lib, dtype, d_in, d_out, T, k, E):
    c = Case(gpu_lib, T, k, E, d_in, d_out, dtype, "swiglu", skew=False)
    c.forward(bias=True, residual=False, pre=True)
    c.dx("gelu")
    c.dw()


def test_nothing_to_sum(gpu_lib):
    """No inputs: y = act(bias) + residual; no rows: empty outputs, and a gradient of zeros."""
    for dtype in TYPES:
        c = Case(gpu_lib, 20, 2, 4, 0, 24, dtype, "silu")
        c.forward(bias=True, residual=True, pre=True)
        c = Case(gpu_lib, 0, 2, 4, 40, 24, dtype, "gelu")
        c.forward(bias=True, residual=True, pre=True)
        c.dx("silu")
        c.dw()
        c = Case(gpu_lib, 30, 2, 4, 40, 24, dtype, "relu", dropped=1.0)
        c.forward(bias=True, residual=True, pre=True)
        c.dx("swiglu")
        c.dw()
        c = Case(gpu_lib, 10, 1, 0, 16, 24, dtype, "none")
        y = torch.full((10, 16), math.nan, dtype=dtype, device="cuda")
        gpu_lib.sptir_moe_product_dx(None, c.dZ_dev[:, :0], c.W_dev[:, :0], y)
        assert (y == 0).all()


def test_residual_may_be_the_output(gpu_lib):
    for dtype, shape in ((BF16, (300, 2, 4, 128, 256)), (F16, (4, 2, 8, 64, 64)), (F32, (70, 2, 3, 33, 51))):
        c = Case(gpu_lib, *shape, dtype, "gelu")
        y = c.residual.cuda()
        gpu_lib.sptir_moe_product(c.r, c.X_dev, c.W_dev, y, residual=y, activation="gelu", gather=True)
        want, limit, _, _ = ref.product(c.parts, c.rows, c.X, c.W, None, c.residual, "gelu")
        ref.check(y, want, limit, "y in place")


@pytest.mark.parametrize("dtype", TYPES)
def test_nan_and_infinity_stay_in_their_rows(gpu_lib, dtype):
    """A row of x that is not finite reaches its own rows of y; an expert's weights reach its own rows; a gradient of an
    expert is not touched by the rows of its neighbours."""
    T, k, E, d_in, d_out = 90, 2, 6, 96, 72
    c = Case(gpu_lib, T, k, E, d_in, d_out, dtype)
    X, W, dZ = c.X.clone(), c.W.clone(), c.dZ.clone()
    X[3, 5], X[7, 0], W[2, 4, 9] = math.nan, math.inf, math.nan
    y = torch.empty(c.rows, d_out, dtype=dtype, device="cuda")
    gpu_lib.sptir_moe_product(c.r, X.cuda(), W.cuda(), y, gather=True)
    ptr, entry, _ = c.order
    expert = torch.bucketize(torch.arange(c.rows), ptr[1:].long(), right=True)
    bad = ((entry // k == 3) | (entry // k == 7))[:, None].expand(-1, d_out).clone()
    bad[:, 4] |= expert == 2
    assert torch.equal(~torch.isfinite(y).cpu(), bad)
    lo, hi = int(ptr[1]), int(ptr[2])
    dZ[lo:hi] = math.nan
    dW, db = torch.empty(E, d_out, d_in, dtype=dtype, device="cuda"), torch.empty(E, d_out, dtype=dtype, device="cuda")
    gpu_lib.sptir_moe_product_dw(c.r, dZ.cuda(), c.X_dev, dW, db=db, gather=True)
    finite = torch.isfinite(dW).all(2).all(1) & torch.isfinite(db).all(1)
    assert finite.cpu().tolist() == [e != 1 for e in range(E)]


def test_product_gradients_against_differences(gpu_lib):
    """Central differences of the forward product in single precision along random directions."""
    T, k, E, d_in, d_out = 60, 2, 5, 40, 56
    for act in ACTS:
        c = Case(gpu_lib, T, k, E, d_in, d_out, F32, act, dropped=0.1, gather=False)
        kept = int(c.order[0][-1])
        X = torch.nan_to_num(c.X)

        def forward(x, w, b):
            y, z = torch.empty(c.rows, d_out, device="cuda"), torch.empty(c.rows, c.wide, device="cuda")
            gpu_lib.sptir_moe_product(c.r, x.cuda(), w.cuda(), y, bias=b.cuda(), pre=z, activation=act)
            return y, z

        y, z = forward(X, c.W, c.bias)
        dY = randn(c.gen, c.rows, d_out).cuda()
        # dZ is the slope's product with dY: the gradient of a product with the identity behind the activation
        eye = torch.eye(d_out, device="cuda").expand(E, d_out, d_out).contiguous()
        dZ = torch.empty(c.rows, c.wide, device="cuda")
        gpu_lib.sptir_moe_product_dx(c.r, dY, eye, dZ, pre=z, activation=act)
        dX, dW, db = torch.empty(c.rows, d_in, device="cuda"), torch.empty_like(c.W, device="cuda"), torch.empty(E, c.wide, device="cuda")
        gpu_lib.sptir_moe_product_dx(c.r, dZ, c.W_dev, dX)
        gpu_lib.sptir_moe_product_dw(c.r, dZ, X.cuda(), dW, db=db)
        h = 2.0 ** -9
        for which in range(3):
            args = [X, c.W, c.bias]
            step = randn(c.gen, *args[which].shape)
            grad = (dX, dW, db)[which].double().cpu()
            lo, hi = list(args), list(args)
            lo[which], hi[which] = args[which] - h * step, args[which] + h * step
            at = [forward(*a)[0].double() for a in (lo, hi)]
            got = float(((at[1] - at[0]) * dY.double())[:kept].sum()) / (2 * h)
            want = float((grad * step.double()).sum())
            # rounding of the values over the step; third derivatives times h^2 (relu: the few that cross 0 within the step)
            size = float((at[0].abs() * dY.double().abs())[:kept].sum()) + float((grad * step.double()).abs().sum())
            curve = 20.0 * float(dY.double().abs().sum()) * (h if act == "relu" else h * h)
            assert abs(got - want) <= 2.0 ** -24 * 16 * size / h + curve, (act, which, got, want)


# ------------------------------------------------------------------------------------------------ how they are called
def layer(lib, logits, X, W1, W2, b, k, bufs, stream=None):
    """The forward of a layer on buffers that are there."""
    E = logits.shape[1]
    lib.sptir_moe_route(logits, bufs["experts"], bufs["weights"], stream=stream)
    r = bufs["routing"] = lib.sptir_moe_sort(bufs["experts"], E, routing=bufs.get("routing"), stream=stream)
    lib.sptir_moe_product(r, X, W1, bufs["h"], bias=b, activation="swiglu", gather=True, stream=stream)
    lib.sptir_moe_product(r, bufs["h"], W2, bufs["ys"], stream=stream)
    lib.sptir_moe_combine(r, bufs["ys"], bufs["y"], weights=bufs["weights"], residual=X, stream=stream)


def layer_inputs(gen, T, E, k, d, f, dtype):
    X, logits = randn(gen, T, d, dtype=dtype).cuda(), randn(gen, T, E, dtype=dtype).cuda()
    W1, W2 = randn(gen, E, 2 * f, d, dtype=dtype, scale=d ** -0.5).cuda(), randn(gen, E, d, f, dtype=dtype, scale=f ** -0.5).cuda()
    b = randn(gen, E, 2 * f, dtype=dtype).cuda()
    bufs = {"experts": torch.empty(T, k, dtype=torch.int32, device="cuda"), "weights": torch.empty(T, k, device="cuda"),
            "h": torch.empty(T * k, f, dtype=dtype, device="cuda"), "ys": torch.empty(T * k, d, dtype=dtype, device="cuda"),
            "y": torch.empty(T, d, dtype=dtype, device="cuda")}
    return logits, X, W1, W2, b, bufs


@pytest.mark.parametrize("T,E,k,d,f", [(1, 16, 4, 256, 128), (200, 8, 2, 192, 320), (20000, 4, 1, 64, 64)])
def test_other_stream_and_capture(gpu_lib, T, E, k, d, f):
    """The same bits on another stream, and from replays of a captured graph with new inputs between them."""
    say("capture", T, E, k, d, f)
    gen = torch.Generator().manual_seed(9)
    logits, X, W1, W2, b, bufs = layer_inputs(gen, T, E, k, d, f, BF16)
    layer(gpu_lib, logits, X, W1, W2, b, k, bufs)
    want = {name: t.clone() for name, t in bufs.items() if name != "routing"}
    for t in want:
        bufs[t].zero_()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    layer(gpu_lib, logits, X, W1, W2, b, k, bufs, stream=side)
    side.synchronize()
    for name, t in want.items():
        assert torch.equal(bufs[name], t), name
    graph = torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        layer(gpu_lib, logits, X, W1, W2, b, k, bufs)
    others = [(logits.clone(), X.clone())] + [(randn(gen, T, E, dtype=BF16).cuda(), randn(gen, T, d, dtype=BF16).cuda()) for _ in range(3)]
    for new_logits, new_X in others:
        logits.copy_(new_logits)
        X.copy_(new_X)
        graph.replay()
        torch.cuda.synchronize()
        got = {name: bufs[name].clone() for name in want}
        eager = layer_inputs(torch.Generator().manual_seed(9), T, E, k, d, f, BF16)[-1]
        layer(gpu_lib, logits, X, W1, W2, b, k, eager)
        torch.cuda.synchronize()
        for name in want:
            assert torch.equal(got[name], eager[name]), name


def test_row_offsets_past_32_bits(gpu_lib):
    """Rows 2^31 elements apart: the last row's offset does not fit 32 bits, in elements or in bytes."""
    T, k, E, d = 3, 1, 2, 64
    apart = 2 ** 31
    gen = torch.Generator().manual_seed(2)
    e = torch.tensor([[1], [0], [1]], dtype=torch.int32)
    r = gpu_lib.sptir_moe_sort(e.cuda(), E)
    far = torch.empty(2 * apart + d, dtype=BF16, device="cuda").as_strided((T, d), (apart, 1))
    X = randn(gen, T, d, dtype=BF16)
    far.copy_(X.cuda())
    Xs = torch.empty(T, d, dtype=BF16, device="cuda")
    gpu_lib.sptir_moe_gather(r, far, Xs)
    assert torch.equal(Xs.cpu(), X[torch.tensor([1, 0, 2])])
    W = randn(gen, E, 64, d, dtype=BF16, scale=0.125)
    near, Y = torch.empty(T, 64, dtype=BF16, device="cuda"), torch.empty(T, 64, dtype=BF16, device="cuda")
    gpu_lib.sptir_moe_product(r, far, W.cuda(), Y, gather=True)
    gpu_lib.sptir_moe_product(r, X.cuda(), W.cuda(), near, gather=True)
    assert torch.equal(Y, near)
    gpu_lib.sptir_moe_product(r, X.cuda(), W.cuda(), far, gather=True)  # (and where it is written)
    assert torch.equal(far, near)
    gpu_lib.sptir_moe_combine(r, far, Y)
    assert torch.equal(Y.cpu(), near.cpu()[torch.tensor([1, 0, 2])])
    dW, dW_near = torch.empty(E, 64, d, dtype=BF16, device="cuda"), torch.empty(E, 64, d, dtype=BF16, device="cuda")
    gpu_lib.sptir_moe_product_dw(r, far, X.cuda(), dW, gather=True)
    gpu_lib.sptir_moe_product_dw(r, near, X.cuda(), dW_near, gather=True)
    assert torch.equal(dW, dW_near)


def test_same_inputs_same_bits(gpu_lib):
    c = Case(gpu_lib, 3000, 2, 5, 256, 192, BF16, "swiglu")
    outs = []
    for _ in range(3):
        y, dW = torch.empty(c.rows, 192, dtype=BF16, device="cuda"), torch.empty_like(c.W_dev)
        db = torch.empty(5, 384, dtype=BF16, device="cuda")
        gpu_lib.sptir_moe_product(c.r, c.X_dev, c.W_dev, y, activation="swiglu", gather=True)
        gpu_lib.sptir_moe_product_dw(c.r, c.dZ_dev, c.X_dev, dW, db=db, gather=True)
        outs.append((y, dW, db))
    for other in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(outs[0], other))


# ------------------------------------------------------------------------------------------------ refusals
def test_refusals(gpu_lib):
    lib = gpu_lib
    dev = dict(device="cuda")
    logits = torch.zeros(4, 8, **dev)
    experts, weights = torch.zeros(4, 2, dtype=torch.int32, **dev), torch.zeros(4, 2, **dev)
    with pytest.raises(TypeError):
        lib.sptir_moe_route(logits.double(), experts, weights)
    with pytest.raises(TypeError):
        lib.sptir_moe_route(logits.cpu(), experts, weights)
    with pytest.raises(TypeError):
        lib.sptir_moe_route(logits, experts.long(), weights)
    with pytest.raises(ValueError):
        lib.sptir_moe_route(logits, experts, weights[:3])
    with pytest.raises(ValueError):
        lib.sptir_moe_route(logits.t(), torch.zeros(8, 2, dtype=torch.int32, **dev), torch.zeros(8, 2, **dev))
    with pytest.raises(lib.SptirError) as e:      # more choices than experts
        lib.sptir_moe_route(logits[:, :1].contiguous(), experts, weights)
    assert e.value.status == 1
    with pytest.raises(lib.SptirError) as e:      # beyond the limits
        lib.sptir_moe_sort(experts, 1025)
    assert e.value.status == 6
    with pytest.raises(lib.SptirError) as e:
        lib.sptir_moe_sort(experts, 0)
    assert e.value.status == 1
    r = lib.sptir_moe_sort(experts, 8)
    with pytest.raises(ValueError):
        lib.sptir_moe_sort(experts, 9, routing=r)
    X, Xs = torch.zeros(4, 16, **dev), torch.zeros(8, 16, **dev)
    with pytest.raises(ValueError):
        lib.sptir_moe_gather(r, X, X)
    with pytest.raises(TypeError):
        lib.sptir_moe_gather(r, X, Xs.half())
    with pytest.raises(ValueError):
        lib.sptir_moe_combine(r, Xs, X, weights=weights[:, :1].contiguous())
    with pytest.raises(ValueError):
        lib.sptir_moe_combine_backward(r, X, None, weights, Xs, weights)
    with pytest.raises(lib.SptirError) as e:      # in place where it cannot be
        lib.sptir_moe_combine_backward(r, X, Xs, weights, Xs, weights)
    assert e.value.status == 1
    W, Y = torch.zeros(8, 24, 16, **dev), torch.zeros(8, 24, **dev)
    with pytest.raises(ValueError):               # X in the order of the tokens needs gather
        lib.sptir_moe_product(r, X, W, Y)
    with pytest.raises(ValueError):
        lib.sptir_moe_product(r, Xs, W, Y, activation="tanh")
    with pytest.raises(ValueError):               # swiglu: half the columns
        lib.sptir_moe_product(r, Xs, W, Y, activation="swiglu")
    with pytest.raises(ValueError):
        lib.sptir_moe_product(r, Xs, W[:7], Y)
    with pytest.raises(ValueError):
        lib.sptir_moe_product(r, Xs, W.transpose(1, 2), Y[:, :16].contiguous())
    with pytest.raises(TypeError):
        lib.sptir_moe_product(r, Xs, W.bfloat16(), Y)
    with pytest.raises(ValueError):
        lib.sptir_moe_product(None, X, W[:1], Y[:4], gather=True)
    with pytest.raises(ValueError):
        lib.sptir_moe_product_dx(r, Y, W, Xs, activation="gelu")
    with pytest.raises(ValueError):
        lib.sptir_moe_product_dw(r, Y, Xs, W[:, :20])
    with pytest.raises(ValueError):               # experts' matrices that overlap
        lib.sptir_moe_product_dw(r, Y, Xs, W, db=torch.zeros(8, 25, **dev))
    shared = torch.zeros(24, 16, **dev).expand(8, 24, 16)
    with pytest.raises(lib.SptirError) as e:
        lib.sptir_moe_product_dw(r, Y, Xs, shared)
    assert e.value.status == 1
    square = torch.zeros(8, 16, 16, **dev)
    with pytest.raises(lib.SptirError) as e:
        lib.sptir_moe_product(r, Xs, square, Xs)
    assert e.value.status == 1
