"""The example layer: all operators in a row, against autograd of the same layer in 64 bits on the values the layer holds."""
import pytest
import torch

import moe_reference as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,experts,top_k,width,hidden", [(1, 8, 2, 64, 32), (50, 6, 2, 72, 40), (400, 16, 4, 128, 96)])
def test_layer_in_single_precision(gpu_lib, tokens, experts, top_k, width, hidden):
    from paper_2207_04606_amd.moe_layer import MoeLayer
    print("[moe layer]", tokens, experts, top_k, width, hidden, flush=True)
    gen = torch.Generator().manual_seed(tokens)
    layer = MoeLayer(tokens, experts, top_k, width, hidden, dtype=torch.float32)
    layer.params["b1"].copy_(torch.randn(experts, 2 * hidden, generator=gen))
    X, dY = torch.randn(tokens, width, generator=gen), torch.randn(tokens, width, generator=gen)
    Y = layer.forward(X.cuda()).clone()
    dX = layer.backward(X.cuda(), dY.cuda())

    p = {name: t.cpu().double().requires_grad_() for name, t in layer.params.items()}
    x = X.double().requires_grad_()
    chosen = layer.experts.cpu().long()
    # (the choice itself: the k largest of the logits that the layer computed)
    assert torch.equal(chosen, ref.route(layer.logits.cpu(), top_k, True)[0].long())
    w = torch.softmax(torch.gather(x @ p["Wr"].t(), 1, chosen), 1)
    y = x
    for j in range(top_k):
        z = torch.matmul(p["W1"][chosen[:, j]], x[:, :, None])[:, :, 0] + p["b1"][chosen[:, j]]
        y = y + w[:, j:j + 1] * torch.matmul(p["W2"][chosen[:, j]], ref.activation(z, "swiglu")[:, :, None])[:, :, 0]
    y.backward(dY.double())

    def near(got, want, what):
        # five products in a row, each of 2^-24 (sqrt(n) + 8) times its terms' size, a few times that of its result
        limit = 2.0 ** -24 * 5 * 8 * (max(width, hidden, tokens) ** 0.5 + 8) * float(want.abs().max())
        err = float((got.cpu().double() - want).abs().max())
        assert err <= limit, (what, err, limit)

    near(Y, y.detach(), "Y")
    near(dX, x.grad, "dX")
    for name in p:
        near(layer.grads[name], p[name].grad, name)


def test_example_learns(gpu_lib, capsys, monkeypatch):
    import re
    import sys

    from paper_2207_04606_amd import moe_layer
    monkeypatch.setattr(sys, "argv", ["moe_layer", "--tokens", "512", "--experts", "8", "--top-k", "2", "--width", "128",
                                      "--hidden", "128", "--steps", "21"])
    torch.manual_seed(0)
    moe_layer.main()
    text = capsys.readouterr().out
    losses = [float(v) for v in re.findall(r"loss ([0-9.]+)", text)]
    assert len(losses) == 3 and losses[-1] < 0.8 * losses[0], text
    assert "one token" in text
