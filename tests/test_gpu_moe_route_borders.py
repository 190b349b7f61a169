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
