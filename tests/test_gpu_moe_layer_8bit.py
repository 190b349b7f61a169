"""The example layer with the grouped router, with activations kept in 8 bits, and in 8-bit integers: the operators in a row, against the
same layer in 64 bits on the values that the layer holds."""
import pytest
import torch

import moe8_reference as ref8
import moe_reference as ref

pytestmark = pytest.mark.gpu

SCORING = {"scores": "sigmoid", "n_groups": 4, "top_groups": 2, "group_top": 2, "normalise": True, "scale": 1.5}


def inputs(tokens, width, experts, hidden, layer, seed):
    gen = torch.Generator().manual_seed(seed)
    layer.params["b1"].copy_(torch.randn(experts, 2 * hidden, generator=gen))
    layer.bias.copy_(0.2 * torch.randn(experts, generator=gen))
    return torch.randn(tokens, width, generator=gen), torch.randn(tokens, width, generator=gen)


@pytest.mark.parametrize("checkpoints", [False, True])
@pytest.mark.parametrize("tokens,experts,top_k,width,hidden", [(1, 8, 2, 64, 32), (50, 8, 3, 72, 40), (400, 16, 4, 128, 96)])
def test_layer_in_single_precision(gpu_lib, checkpoints, tokens, experts, top_k, width, hidden):
    from paper_2207_04606_amd.moe_layer import MoeLayer
    print("[moe layer]", checkpoints, tokens, experts, top_k, width, hidden, flush=True)
    layer = MoeLayer(tokens, experts, top_k, width, hidden, dtype=torch.float32, scoring=SCORING, checkpoints=checkpoints)
    X, dY = inputs(tokens, width, experts, hidden, layer, tokens)
    Y = layer.forward(X.cuda()).clone()
    z_kept = layer.pre.cpu()
    dX = layer.backward(X.cuda(), dY.cuda())

    p = {name: t.cpu().double().requires_grad_() for name, t in layer.params.items()}
    x = X.double().requires_grad_()
    chosen = layer.experts.cpu().long()
    assert torch.equal(chosen, ref8.route(layer.logits.cpu(), top_k, bias=layer.bias.cpu(), **SCORING)[0].long())

    # what the gradients read of x and z is what was kept of them; their values go on unchanged
    class Reads(torch.autograd.Function):
        @staticmethod
        def forward(ctx, values, kept):
            return kept

        @staticmethod
        def backward(ctx, d):
            return d, None

    slot = layer.routing.slot_of.cpu().view(tokens, top_k).long()
    x_read = x
    if checkpoints:
        x_read = Reads.apply(x, ref8.kept(*ref8.pack(X), torch.float32).double())
        z_of = ref8.kept(*ref8.pack(z_kept), torch.float32).double()
    s = torch.sigmoid(torch.gather(x @ p["Wr"].t(), 1, chosen))
    w = 1.5 * s / s.sum(1, keepdim=True)
    y, total = x, torch.zeros((), dtype=torch.float64)
    for j in range(top_k):
        z = torch.matmul(p["W1"][chosen[:, j]], x[:, :, None])[:, :, 0] + p["b1"][chosen[:, j]]
        y = y + w[:, j:j + 1] * torch.matmul(p["W2"][chosen[:, j]], ref.activation(z, "swiglu")[:, :, None])[:, :, 0]
        if checkpoints:  # <dY, w ys> whose gradients are those of the kept values: the router's through ys as it was, the experts' through z as it is kept
            ys = torch.matmul(p["W2"][chosen[:, j]], ref.activation(z, "swiglu")[:, :, None])[:, :, 0].detach()
            zk = torch.matmul(p["W1"][chosen[:, j]], x_read[:, :, None])[:, :, 0] + p["b1"][chosen[:, j]]
            yk = torch.matmul(p["W2"][chosen[:, j]], ref.activation(Reads.apply(zk, z_of[slot[:, j]]), "swiglu")[:, :, None])[:, :, 0]
            total = total + (dY.double() * (w[:, j:j + 1] * ys + w[:, j:j + 1].detach() * yk)).sum()
    if checkpoints:
        (total + (dY.double() * x).sum()).backward()
    else:
        y.backward(dY.double())

    def near(got, want, what):
        # five products in a row, each of 2^-24 (sqrt(n) + 8) times its terms' size, a few times that of its result (what is kept is that of
        # the layer's own z, so no code differs)
        limit = 2.0 ** -24 * 5 * 8 * (max(width, hidden, tokens) ** 0.5 + 8) * float(want.abs().max())
        err = float((got.cpu().double() - want).abs().max())
        assert err <= limit, (what, err, limit)

    near(Y, y.detach(), "Y")
    near(dX, x.grad, "dX")
    for name in p:
        near(layer.grads[name], p[name].grad, name)


def test_what_is_kept_is_close_in_bf16(gpu_lib):
    """Gradients with and without checkpoints differ by what 8 bits leave of x and z: a code is off by its unit over the root of 12 on average, and
    a unit is at most a 64th of the block's largest, some 2.5 times a value's size: 2.5 / 64 / 3.5, 1.1 % of it.  A gradient has that once from x or from
    the slope at z, whose own relative change is up to twice that of z: below 2^-5 in all."""
    from paper_2207_04606_amd.moe_layer import MoeLayer
    sizes = (512, 8, 2, 128, 96)
    layers = [MoeLayer(*sizes, scoring=SCORING, checkpoints=c, seed=5) for c in (False, True)]
    X, dY = inputs(512, 128, 8, 96, layers[0], 3)
    inputs(512, 128, 8, 96, layers[1], 3)
    X, dY = X.cuda().bfloat16(), dY.cuda().bfloat16()
    results = []
    for layer in layers:
        layer.forward(X)
        dX = layer.backward(X, dY).clone()
        results.append([dX, *(layer.grads[name].clone() for name in sorted(layer.grads))])
    for a, b in zip(*results):
        assert torch.isfinite(b).all()
        assert float((a.double() - b.double()).norm()) <= 2.0 ** -5 * float(a.double().norm())


@pytest.mark.parametrize("tokens,experts,top_k,width,hidden", [(1, 8, 2, 64, 32), (50, 8, 3, 72, 40), (700, 16, 4, 128, 96)])
def test_layer_in_8_bit_integers(gpu_lib, tokens, experts, top_k, width, hidden):
    from paper_2207_04606_amd.moe_layer import Int8MoeLayer, MoeLayer
    layer = MoeLayer(1, experts, top_k, width, hidden, dtype=torch.float32, scoring=SCORING, train=False)
    X, _ = inputs(tokens, width, experts, hidden, layer, tokens + 1)
    answers = Int8MoeLayer(layer, tokens)
    Y = answers.forward(X.cuda()).cpu()
    chosen, w = answers.experts.cpu().long(), answers.weights.cpu().double()
    want_e, want_w = ref8.route(answers.logits.cpu(), top_k, bias=layer.bias.cpu(), **SCORING)
    assert torch.equal(chosen, want_e.long())

    def dequantised(codes, scales):
        return codes.double() * scales.double()[..., None]

    W1, W2 = (dequantised(*ref8.quantise(layer.params[n].cpu().view(-1, layer.params[n].shape[2]))).view(layer.params[n].shape) for n in ("W1", "W2"))
    x8 = dequantised(*ref8.quantise(X))
    h8 = dequantised(*ref8.quantise(answers.h.cpu()))      # (of the h that the layer has)
    slot = answers.routing.slot_of.cpu().view(tokens, top_k).long()
    y = X.double()
    size = torch.zeros_like(y)
    for j in range(top_k):
        z = torch.matmul(W1[chosen[:, j]], x8[:, :, None])[:, :, 0] + layer.params["b1"].cpu().double()[chosen[:, j]]
        h = ref.activation(z, "swiglu")
        got = answers.h.cpu().double()[slot[:, j]]
        assert float((got - h).abs().max()) <= 2.0 ** -19 * float(z.abs().max()) ** 2
        part = w[:, j:j + 1] * torch.matmul(W2[chosen[:, j]], h8[slot[:, j]][:, :, None])[:, :, 0]
        y, size = y + part, size + part.abs()
    # a scaled whole number (three roundings), times a weight, top_k + 1 terms
    assert ((Y.double() - y).abs() <= 2.0 ** -24 * (top_k + 8) * (size + y.abs())).all()
