"""The grouped router where float32 cannot say, or 16-bit logits cannot stand for their scores: it has to notice.  Choices against the definition in
64 bits (moe8_reference.route), exactly."""
import math

import pytest
import torch

import moe8_reference as ref8
import moe_reference as ref
from test_gpu_moe import BF16, F16, F32, TYPES, randn, say
from test_gpu_moe_route_groups import run

pytestmark = pytest.mark.gpu

GROUPS = [(1, 1, 1), (8, 3, 1), (8, 3, 2)]


def same(lib, l, k, bias=None, **how):
    how = {"normalise": True, "scale": 1.0, **how}
    want, w_want = ref8.route(l, k, bias=bias, **how)
    _, experts, weights = run(lib, l, k, bias=None if bias is None else bias.cuda(), **how)
    off = (experts.cpu() != want).any(1)
    assert not off.any(), f"{int(off.sum())} of {len(off)} tokens, the first {int(off.nonzero()[0])}"
    # (computed in float64 and rounded once)
    ref.check(weights, w_want, w_want.abs() * 2.0 ** -24 * 1.01 + 2.0 ** -149, "weights")


# ------------------------------------------------------------------------------------------------ sums of a group's two largest
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scores", ["sigmoid", "softmax"])
@pytest.mark.parametrize("E,n_groups,top_groups,k", [(32, 8, 3, 4), (60, 6, 2, 3), (6, 3, 1, 1), (256, 8, 4, 8), (512, 16, 5, 6)])
def test_groups_of_scores_near_the_smallest(gpu_lib, dtype, scores, E, n_groups, top_groups, k):
    """Scores around 2^-100, of which some are cut off where float32's keys end: what was cut off is no part of a sum."""
    say("small groups", dtype, scores, E, n_groups, top_groups, k)
    gen = torch.Generator().manual_seed(E)
    T = 400
    l = -100.0 * math.log(2.0) + randn(gen, T, E, scale=1.5)
    l[torch.rand(T, E, generator=gen) < 0.3] = -90.0
    l[torch.rand(T, E, generator=gen) < 0.3] = -math.inf
    l[200:] -= 0.7
    if scores == "softmax":
        l[:, 0] = 0.0                                      # (the others' scores are exp of their logits)
    same(gpu_lib, l.to(dtype), k, scores=scores, n_groups=n_groups, top_groups=top_groups, group_top=2)


@pytest.mark.parametrize("scores", ["sigmoid", "softmax"])
def test_one_small_score_beside_two(gpu_lib, scores):
    """1.5 * 2^-100 alone in its group, more than 1.01 * 2^-100 beside 2^-130."""
    ln2 = math.log(2.0)
    l = torch.tensor([[0.0, -1.0, -99.99 * ln2, -130.0 * ln2, -99.4 * ln2, -math.inf, -99.98 * ln2, -131.0 * ln2]])
    if scores == "sigmoid":
        l[0, :2] = -98.0 * ln2
    same(gpu_lib, l, 3, scores=scores, n_groups=4, top_groups=2, group_top=2)


@pytest.mark.parametrize("scores", ["sigmoid", "softmax"])
def test_groups_of_biases_past_the_keys(gpu_lib, scores):
    """Biases beyond 2^90, where float32's keys are cut off, in sums with others: 2^91.5 - 2^91 is more than 2^75."""
    big, off = [2.0 ** 91.5, -2.0 ** 91.0], -2.0 ** 100
    cases = [([2.0 ** 75, 0.0, *big, 0.0, 0.0], 3, 1, 1), ([2.0 ** 70, 0.0, 2.0 ** 79.9, -2.0 ** 95, 0.0, -2.0 ** 90 * (1 - 2.0 ** -12), off, off], 4, 2, 1),
             ([0.0, off, 0.1, 2 * off, 0.2, 4 * off, -0.1, off], 4, 2, 2), ([0.5, -3e38, 0.25, -3e38, 0.0, 0.0, 1e30, -1e31], 4, 2, 2),
             ([2.0 ** 80, 2.0 ** 79, 2.0 ** 80, 2.0 ** 79.5, -2.0 ** 88, 2.0 ** 81, 1.0, 1.0], 4, 2, 2)]
    gen = torch.Generator().manual_seed(7)
    for bias, n_groups, top_groups, k in cases:
        bias = torch.tensor(bias)
        l = torch.cat([torch.zeros(1, len(bias)), randn(gen, 20, len(bias))])
        same(gpu_lib, l, k, bias=bias, scores=scores, n_groups=n_groups, top_groups=top_groups, group_top=2)
    for each in (2, 3, 8):
        bias = torch.sign(randn(gen, 8 * each)) * torch.exp2(60.0 + 60.0 * torch.rand(8 * each, generator=gen))
        bias[torch.rand(8 * each, generator=gen) < 0.5] = 0.0
        same(gpu_lib, randn(gen, 50, 8 * each), 2, bias=bias, scores=scores, n_groups=8, top_groups=3, group_top=2)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scores", ["sigmoid", "softmax"])
@pytest.mark.parametrize("group_top", [1, 2])
def test_padding_beside_other_tokens(gpu_lib, dtype, scores, group_top):
    """Tokens without any candidate, in every place of a wavefront, beside some with as many groups as stay and fewer."""
    gen = torch.Generator().manual_seed(group_top)
    T, E, G = 300, 64, 8
    l = randn(gen, T, E, scale=2.0)
    for t in range(T):
        for g in range(G):
            if (t * 7 + g * 3) % 8 < t % 9:
                l[t, g * 8:g * 8 + 8] = -math.inf
    for bias in (None, 0.1 * randn(gen, E)):
        same(gpu_lib, l.to(dtype), 4, bias=bias, scores=scores, n_groups=G, top_groups=3, group_top=group_top)


# ------------------------------------------------------------------------------------------------ 16-bit logits as keys
@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("n_groups,top_groups,group_top", GROUPS)
def test_sigmoids_next_to_one(gpu_lib, dtype, n_groups, top_groups, group_top):
    """Past 37 all sigmoids are 1 in float64, and ties go to the lower id, where the larger logits have the higher ones."""
    gen = torch.Generator().manual_seed(n_groups + group_top)
    T, E = 200, 64
    l = torch.sort(28.0 + 32.0 * torch.rand(T, E, generator=gen), dim=1)[0]
    l[50:100] = 36.0 + 24.0 * torch.rand(50, E, generator=gen)
    l[100:150, :48] = randn(gen, 50, 48)                   # few next to one
    l[150:] = randn(gen, 50, E, scale=40.0)
    same(gpu_lib, l.to(dtype), 6, scores="sigmoid", n_groups=n_groups, top_groups=top_groups, group_top=group_top)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("scores", ["sigmoid", "softmax"])
@pytest.mark.parametrize("n_groups,top_groups,group_top", GROUPS)
def test_logits_next_to_zero(gpu_lib, dtype, scores, n_groups, top_groups, group_top):
    """Logits whose scores are one number in float64 (below 2^-55: every exponential is 1 and every sigmoid 1/2), subnormal ones and both zeros among them,
    and logits around 2^-36, whose scores float64 tells apart where their type does: by 2^-45 at least, 2^-53 being float64's unit there."""
    gen = torch.Generator().manual_seed(n_groups)
    T, E = 120, 64
    tiny = torch.finfo(dtype).smallest_normal
    kinds = [torch.sign(randn(gen, T // 3, E)) * (2.0 ** -70 if dtype is not F16 else 0.0) * (1.0 + torch.rand(T // 3, E, generator=gen)),
             randn(gen, T // 3, E, scale=tiny / 4) if dtype is not F16 else torch.sign(randn(gen, T // 3, E)) * 0.0,
             torch.sign(randn(gen, T // 3, E)) * 2.0 ** (-36 if dtype is not F16 else -20) * (1.0 + torch.round(64 * torch.rand(T // 3, E, generator=gen)) / 64)]
    if group_top == 2:
        kinds.pop()                                        # (sums of different scores that differ in the last place, if at all)
    l = torch.cat(kinds).to(dtype)
    l[::5] = torch.sort(l[::5].float(), dim=1)[0].to(dtype)  # (the larger ones at the higher ids)
    same(gpu_lib, l, 6, scores=scores, n_groups=n_groups, top_groups=top_groups, group_top=group_top)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("scores", ["sigmoid", "softmax"])
@pytest.mark.parametrize("n_groups,top_groups,group_top", GROUPS)
def test_more_equal_logits_than_choices(gpu_lib, dtype, scores, n_groups, top_groups, group_top):
    """The last choice is one of many equal logits, and others that are smaller have its score and lower ids: zeros of the other sign, 0 beside 2^-70."""
    E = 64
    rows = []
    for most, few in ((0.0, -0.0), (-0.0, 0.0), (2.0 ** -70, 0.0), (2.0 ** -70, -0.0), (0.0, -2.0 ** -70), (2.0 ** -70, 2.0 ** -71), (2.0 ** -24, 0.0), (1.0, 0.5),
                      (0.0, -2.0 ** -24), (2.0 ** -27, 2.0 ** -28), (2.0 ** -60, 2.0 ** -130)):
        for first in (0, 1, 8, 19):
            l = torch.full((E,), most)
            l[first:first + 8] = few                       # (a whole group, and parts of two)
            if first == 1:
                l[40:] = 3.0
                l[50] = few
            rows.append(l)
    same(gpu_lib, torch.stack(rows).to(dtype), 6, scores=scores, n_groups=n_groups, top_groups=top_groups, group_top=group_top)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("n_groups,top_groups,group_top", GROUPS)
def test_softmaxes_that_float64_cannot_hold(gpu_lib, dtype, n_groups, top_groups, group_top):
    """Exponents of -600 and beyond: of those below -750 nothing is left, and they tie."""
    gen = torch.Generator().manual_seed(n_groups)
    T, E = 120, 64
    l = -500.0 - 400.0 * torch.rand(T, E, generator=gen)
    l[40:80] = -760.0 - 400.0 * torch.rand(40, E, generator=gen)
    l[80:] *= 60.0
    # (none whose exponential has few digits left: one more or less of them is the last place of the library's)
    l = torch.where((l < -700.0) & (l > -750.0), -650.0, l)
    l = torch.sort(l, dim=1)[0]
    l[:, 5] = 0.0
    same(gpu_lib, l.to(dtype), 6, scores="softmax", n_groups=n_groups, top_groups=top_groups, group_top=group_top)
