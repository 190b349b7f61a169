"""The grouped router against its definition in 64 bits (tests/moe8_reference.py): scores, bias, groups, ties, masks, types, strides, values
at the ends of their types, gradients."""
import math

import pytest
import torch

import moe8_reference as ref8
import moe_reference as ref
from test_gpu_moe import TYPES, masked_logits, out_like, randn, say, strided

pytestmark = pytest.mark.gpu

# tokens, experts, choices, groups, of which stay, whose score is the sum of so many, columns behind the logits
SHAPES = [(1, 1, 1, 1, 1, 1, 0), (1, 256, 8, 8, 4, 2, 0), (5, 6, 2, 3, 2, 2, 5), (37, 8, 2, 4, 1, 1, 0), (70, 60, 6, 6, 3, 1, 4), (129, 66, 64, 33, 32, 2, 1),
          (64, 128, 8, 1, 1, 1, 0), (33, 200, 7, 8, 3, 2, 3), (300, 16, 4, 16, 5, 2, 0), (9, 1000, 16, 40, 2, 2, 0), (6, 1024, 1, 64, 64, 1, 8),
          (40, 64, 5, 64, 9, 2, 0), (65, 256, 16, 2, 1, 2, 0)]


def biases(gen, E, scores):
    b = randn(gen, E, scale=0.3 if scores == "sigmoid" else 2.0 / E)
    b[::3] = b[0]                                          # ties of experts with the same logits
    if E > 8:
        b[5] = -math.inf                                   # switched off
        b[7] = math.nan
    return b


def run(lib, l, k, extra=0, **how):
    T = l.shape[0]
    dev = strided(l, extra)
    experts = torch.full((T, k), -7, dtype=torch.int32, device="cuda")
    weights = torch.full((T, k), math.nan, device="cuda")
    lib.sptir_moe_route_groups(dev, experts, weights, **how)
    return dev, experts, weights


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("normalise,scale,with_bias", [(True, 2.5, True), (False, 1.0, False), (False, -0.75, True), (True, 1.0, False)])
@pytest.mark.parametrize("T,E,k,n_groups,top_groups,group_top,extra", SHAPES)
def test_route_groups(gpu_lib, dtype, scores, normalise, scale, with_bias, T, E, k, n_groups, top_groups, group_top, extra):
    say("route groups", dtype, scores, normalise, T, E, k, n_groups, top_groups, group_top)
    gen = torch.Generator().manual_seed(T * 1000 + E + k)
    l = masked_logits(gen, T, E, dtype)
    bias = biases(gen, E, scores) if with_bias else None
    how = {"scores": scores, "n_groups": n_groups, "top_groups": top_groups, "group_top": group_top, "normalise": normalise, "scale": scale}
    want, w_want = ref8.route(l, k, bias=bias, **how)
    dev, experts, weights = run(gpu_lib, l, k, extra, bias=None if bias is None else bias.cuda(), **how)
    assert torch.equal(experts.cpu(), want)
    # computed in float64 and rounded once; the sum under a softmax that is not normalised is one of float32 exponentials: each within 2^-23 of
    # its own and, for the rounding of its exponent d, d 2^-24, whose mean under the softmax is its entropy less the log of the sum: below log E
    near = 1.01 if scores == "sigmoid" or normalise else 1.01 + 2.0 + math.log(E)
    ref.check(weights, w_want, w_want.abs() * 2.0 ** -24 * near + 2.0 ** -149, "weights")
    dw = randn(gen, T, k)
    dw[want < 0] = math.nan                                # of a choice that is none
    want_d = ref8.route_gradient(l, want, dw, scores, normalise, scale)
    d, rest = out_like(T, E, dtype, extra)
    gpu_lib.sptir_moe_route_groups_backward(dev, experts, weights, dw.cuda(), d, scores=scores, normalise=normalise, scale=scale)
    # as sptir_moe_route_backward: softmax of differences below 200, sums over experts and choices, a sigmoid
    size = float(torch.where(want < 0, torch.zeros_like(dw), dw).abs().max()) * 2 * abs(scale)
    limit = 1.01 * ref.UNIT[dtype] * want_d.abs() + size * (2.0 ** -24 * 200.0 + (math.sqrt(E) + k + 16) * 2.0 ** -22) + ref.TINY[dtype]
    ref.check(d, want_d, limit, "d_logits")
    assert torch.isnan(rest).all()


@pytest.mark.parametrize("normalise", [True, False])
@pytest.mark.parametrize("T,E,k", [(1, 64, 8), (70, 60, 6), (33, 200, 7), (9, 1000, 16)])
def test_softmax_without_bias_or_groups_is_the_plain_router(gpu_lib, T, E, k, normalise):
    gen = torch.Generator().manual_seed(E)
    l = randn(gen, T, E, scale=2.0)
    _, experts, weights = run(gpu_lib, l, k, normalise=normalise)
    e2, w2 = torch.empty_like(experts), torch.empty_like(weights)
    gpu_lib.sptir_moe_route(l.cuda(), e2, w2, normalise=normalise)
    assert torch.equal(experts, e2)
    assert float((weights - w2).abs().max()) <= 2.0 ** -24 * 200.0


def test_keys_closer_than_float32(gpu_lib):
    """c that float32 rounds to one number, in every place of a token's lanes: the order is that of 64 bits."""
    E, k, T = 256, 16, 64
    gen = torch.Generator().manual_seed(0)
    # sigmoids of -30 +- are 1e-13 apart beside a bias of 1
    l = -30.0 + randn(gen, T, E, scale=2.0)
    bias = torch.ones(E)
    for n_groups, top_groups in ((1, 1), (8, 3)):
        how = {"scores": "sigmoid", "n_groups": n_groups, "top_groups": top_groups, "group_top": 2, "normalise": True, "scale": 1.0}
        want, w_want = ref8.route(l, k, bias=bias, **how)
        _, experts, weights = run(gpu_lib, l, k, bias=bias.cuda(), **how)
        assert torch.equal(experts.cpu(), want)
        ref.check(weights, w_want, w_want * 2.0 ** -23, "weights")


def test_values_at_the_ends(gpu_lib):
    """Sigmoids that float32 or float64 cannot hold are normalised all the same; infinities and NaN reach their own token only."""
    low, inf, nan = torch.finfo(torch.float32).min, math.inf, math.nan
    l = torch.tensor([[-200.0, -201.0, -300.0, -400.0], [low, low, low, low], [-1000.0, -1001.0, low, -inf], [inf, 1.0, 0.0, -1.0],
                      [nan, 1.0, 0.0, -1.0], [-inf, -inf, -inf, -inf], [200.0, 300.0, 100.0, 0.0]])
    _, experts, weights = run(gpu_lib, l, 2, scores="sigmoid")
    assert experts.cpu().tolist() == [[0, 1], [0, 1], [0, 1], [0, 1], [1, 2], [-1, -1], [0, 1]]
    w = weights.cpu().double()
    assert torch.isfinite(w).all()
    e = math.exp(-1.0)
    for row, want in ((0, [1 / (1 + e), e / (1 + e)]), (1, [0.5, 0.5]), (2, [1 / (1 + e), e / (1 + e)]), (5, [0.0, 0.0]), (6, [0.5, 0.5])):
        assert float((w[row] - torch.tensor(want)).abs().max()) <= 2.0 ** -24
    d = torch.empty(7, 4, device="cuda")
    gpu_lib.sptir_moe_route_groups_backward(l.cuda(), experts, weights, torch.ones(7, 2, device="cuda"), d, scores="sigmoid")
    assert torch.isfinite(d).all()
    for normalise in (True, False):
        _, experts, weights = run(gpu_lib, l, 2, scores="softmax", normalise=normalise)
        assert experts.cpu()[3].tolist() == [0, 1] and experts.cpu()[4].tolist() == [1, 2]
        w = weights.cpu()
        assert torch.isnan(w[3, 0]) and torch.isfinite(w[[0, 1, 2, 5, 6]]).all()
        assert torch.isnan(w[4]).all() == (not normalise)


@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("normalise", [True, False])
def test_gradient_against_differences(gpu_lib, scores, normalise):
    T, E, k, step = 40, 24, 3, 2.0 ** -6
    gen = torch.Generator().manual_seed(3)
    # logits of a token at least 8 steps apart, so that a step changes no choice
    l = torch.stack([torch.randperm(E, generator=gen) for _ in range(T)]).float() * 0.125
    dw, direction = randn(gen, T, k).cuda(), torch.sign(randn(gen, T, E)).cuda()
    how = {"scores": scores, "normalise": normalise, "scale": 1.5}
    _, experts, weights = run(gpu_lib, l, k, n_groups=4, top_groups=4, **how)
    l = l.cuda()
    d = torch.empty_like(l)
    gpu_lib.sptir_moe_route_groups_backward(l, experts, weights, dw, d, **how)
    ends = []
    for sign in (-1.0, 1.0):
        e = torch.empty_like(experts)
        w = torch.empty_like(weights)
        gpu_lib.sptir_moe_route_groups(l + sign * step * direction, e, w, **how)
        assert torch.equal(e, experts)
        ends.append(w.double())
    slope = ((ends[1] - ends[0]) * dw.double()).sum(1) / (2 * step)
    want = (d.double() * direction.double()).sum(1)
    # third derivative of a softmax entry or of a sigmoid along a sign vector: below 8; two float32 weights over the step
    limit = 1.5 * dw.double().abs().sum(1) * (8 * step ** 2 / 6 + 2.0 ** -22 / step)
    assert ((slope - want).abs() <= limit).all()


def test_more_tokens_than_a_launch_takes(gpu_lib):
    """2^25 tokens and a few: the last ones and those at the border."""
    T, E, k = (1 << 25) + 5, 4, 2
    l = torch.empty(T, E, dtype=torch.bfloat16, device="cuda").normal_()
    bias = torch.tensor([0.1, -0.1, 0.3, 0.0], device="cuda")
    experts = torch.full((T, k), -7, dtype=torch.int32, device="cuda")
    weights = torch.full((T, k), math.nan, device="cuda")
    how = {"scores": "sigmoid", "n_groups": 2, "top_groups": 1, "group_top": 2}
    gpu_lib.sptir_moe_route_groups(l, experts, weights, bias=bias, **how)
    assert int(experts.amin()) >= 0 and bool(torch.isfinite(weights).all())
    d = torch.full((T, E), math.nan, dtype=torch.bfloat16, device="cuda")
    gpu_lib.sptir_moe_route_groups_backward(l, experts, weights, torch.ones_like(weights), d, scores="sigmoid")
    assert bool(torch.isfinite(d).all())
    for at in (slice(0, 64), slice((1 << 25) - 32, T)):
        want, w_want = ref8.route(l[at].cpu(), k, bias=bias.cpu(), normalise=True, scale=1.0, **how)
        assert torch.equal(experts[at].cpu(), want)
        ref.check(weights[at], w_want, w_want * 2.0 ** -23, "weights")


@pytest.mark.parametrize("scores", ["sigmoid", "softmax"])
def test_in_a_graph(gpu_lib, scores):
    T, E, k = 300, 64, 4
    gen = torch.Generator().manual_seed(8)
    inputs = [randn(gen, T, E).cuda() for _ in range(3)]
    bias, dw = (0.1 * randn(gen, E)).cuda(), randn(gen, T, k).cuda()
    l, d = inputs[0].clone(), torch.empty(T, E, device="cuda")
    experts, weights = torch.empty(T, k, dtype=torch.int32, device="cuda"), torch.empty(T, k, device="cuda")

    def step(stream=None):
        gpu_lib.sptir_moe_route_groups(l, experts, weights, scores=scores, bias=bias, n_groups=8, top_groups=3, group_top=2, stream=stream)
        gpu_lib.sptir_moe_route_groups_backward(l, experts, weights, dw, d, scores=scores, stream=stream)

    want = []
    for x in inputs:
        l.copy_(x)
        step()
        want.append([t.clone() for t in (experts, weights, d)])
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step()
    for n in range(6):
        l.copy_(inputs[n % 3])
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip((experts, weights, d), want[n % 3]))
        inputs[0].sum().item()
        d.fill_(math.nan)
        side.wait_stream(torch.cuda.current_stream())
        step(side)
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip((experts, weights, d), want[n % 3]))


def test_refusals(gpu_lib):
    l = torch.zeros(4, 12, device="cuda")
    e, w = torch.empty(4, 2, dtype=torch.int32, device="cuda"), torch.empty(4, 2, device="cuda")
    for how in ({"scores": "tanh"}, {"bias": torch.zeros(11, device="cuda")}):
        with pytest.raises(ValueError):
            gpu_lib.sptir_moe_route_groups(l, e, w, **how)
    with pytest.raises(TypeError):
        gpu_lib.sptir_moe_route_groups(l, e, w, bias=torch.zeros(12, dtype=torch.float16, device="cuda"))
    for how, status in (({"n_groups": 5}, 1), ({"n_groups": 0}, 1), ({"n_groups": 4, "top_groups": 5}, 1), ({"n_groups": 4, "top_groups": 0}, 1),
                        ({"group_top": 0}, 1), ({"group_top": 3}, None), ({"n_groups": 12, "top_groups": 1}, 1), ({"scale": math.inf}, 1), ({"scale": math.nan}, 1)):
        with pytest.raises(gpu_lib.SptirError) as caught:
            gpu_lib.sptir_moe_route_groups(l, e, w, **how)
        assert status is None or caught.value.status == status
