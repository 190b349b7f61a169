"""A mixture-of-experts layer on the library's operators: forward, backward, and the forward of single tokens.

`MoeLayer` keeps the buffers of one size of batch, as a training or serving program does, and runs

    logits = X Wr^T                                   (dense product)
    experts, weights = the k largest logits, softmax  (sptir_moe_route), entries sorted by expert (sptir_moe_sort)
    h[s]  = silu(gate) * up of W1[e] x + b1[e]        (sptir_moe_product, x gathered by it)
    ys[s] = W2[e] h[s]
    Y[t]  = X[t] + sum_j weights[t, j] ys[slot(t, j)] (sptir_moe_combine)

and its gradients.  Run as

    python3 -m paper_2207_04606_amd.moe_layer [--tokens 8192] [--experts 32] [--top-k 4] [--width 1024] [--hidden 1024]

it trains the layer for a few steps towards the outputs of another one of the same form, prints the loss, and then times a
training step and the forward of one token (eagerly, and as a replayed graph).
"""
from __future__ import annotations

import argparse

import torch

from . import moe


class MoeLayer:
    def __init__(self, tokens, experts, top_k, width, hidden, dtype=torch.bfloat16, train=True, seed=0, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)

        def matrix(*shape):
            return (torch.randn(*shape, generator=gen, device=device) * shape[-1] ** -0.5).to(dtype)

        def empty(*shape, dtype=dtype):
            return torch.empty(*shape, dtype=dtype, device=device)

        n = tokens * top_k
        self.top_k, self.n_experts, self.train = top_k, experts, train
        self.params = {"Wr": matrix(experts, width), "W1": matrix(experts, 2 * hidden, width),
                       "b1": torch.zeros(experts, 2 * hidden, dtype=dtype, device=device), "W2": matrix(experts, width, hidden)}
        self.logits, self.experts = empty(tokens, experts), empty(tokens, top_k, dtype=torch.int32)
        self.weights = empty(tokens, top_k, dtype=torch.float32)
        self.h, self.ys, self.Y = empty(n, hidden), empty(n, width), empty(tokens, width)
        self.routing = None
        if train:
            self.pre, self.d_ys, self.d_pre, self.dx = empty(n, 2 * hidden), empty(n, width), empty(n, 2 * hidden), empty(n, width)
            self.d_weights, self.d_logits, self.dX_router = torch.empty_like(self.weights), torch.empty_like(self.logits), empty(tokens, width)
            self.dX = empty(tokens, width)
            self.grads = {name: torch.empty_like(p) for name, p in self.params.items()}

    def forward(self, X):
        p = self.params
        moe.sptir_moe_product(None, X, p["Wr"], self.logits)
        moe.sptir_moe_route(self.logits, self.experts, self.weights)
        r = self.routing = moe.sptir_moe_sort(self.experts, self.n_experts, routing=self.routing)
        moe.sptir_moe_product(r, X, p["W1"], self.h, bias=p["b1"], activation="swiglu", gather=True,
                              pre=self.pre if self.train else None)
        moe.sptir_moe_product(r, self.h, p["W2"], self.ys)
        moe.sptir_moe_combine(r, self.ys, self.Y, weights=self.weights, residual=X)
        return self.Y

    def backward(self, X, dY):
        """Gradients of the parameters (self.grads) and of X, after forward(X)."""
        p, g, r = self.params, self.grads, self.routing
        moe.sptir_moe_combine_backward(r, dY, self.ys, self.weights, self.d_ys, self.d_weights)
        moe.sptir_moe_product_dw(r, self.d_ys, self.h, g["W2"])
        moe.sptir_moe_product_dx(r, self.d_ys, p["W2"], self.d_pre, pre=self.pre, activation="swiglu")
        moe.sptir_moe_product_dw(r, self.d_pre, X, g["W1"], db=g["b1"], gather=True)
        moe.sptir_moe_product_dx(r, self.d_pre, p["W1"], self.dx)
        moe.sptir_moe_route_backward(self.logits, self.experts, self.weights, self.d_weights, self.d_logits)
        moe.sptir_moe_product_dw(None, self.d_logits, X, g["Wr"])
        moe.sptir_moe_product_dx(None, self.d_logits, p["Wr"], self.dX_router)
        # X reaches Y through its entries, the router and the residual
        self.dX_router += dY
        moe.sptir_moe_combine(r, self.dx, self.dX, residual=self.dX_router)
        return self.dX


def _timed(fn, reps):
    for _ in range(3):
        fn()
    torch.cuda.synchronize()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    for _ in range(reps):
        fn()
    e1.record()
    torch.cuda.synchronize()
    return e0.elapsed_time(e1) / reps


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=8192)
    ap.add_argument("--experts", type=int, default=32)
    ap.add_argument("--top-k", type=int, default=4)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--rate", type=float, default=0.5)
    a = ap.parse_args()
    sizes = (a.experts, a.top_k, a.width, a.hidden)
    layer, goal = MoeLayer(a.tokens, *sizes, seed=1), MoeLayer(a.tokens, *sizes, train=False, seed=2)
    goal.params["W2"] *= 0.5
    X = torch.randn(a.tokens, a.width, device="cuda").bfloat16()
    target = goal.forward(X).float()
    master = {name: p.float() for name, p in layer.params.items()}
    for step in range(a.steps):
        diff = layer.forward(X).float() - target
        layer.backward(X, (diff / a.tokens).bfloat16())
        for name, p in layer.params.items():
            # (an expert sees a share of the tokens)
            master[name] -= a.rate * (a.experts / a.top_k if name != "Wr" else 1.0) * layer.grads[name].float()
            p.copy_(master[name])
        if step % 10 == 0 or step == a.steps - 1:
            print(f"step {step}: loss {0.5 * float((diff * diff).sum()) / a.tokens:.4f}", flush=True)
    dY = torch.randn_like(X)
    print(f"forward {_timed(lambda: layer.forward(X), 10):.3f} ms, with backward "
          f"{_timed(lambda: (layer.forward(X), layer.backward(X, dY)), 10):.3f} ms ({a.tokens} tokens)")
    one = MoeLayer(1, *sizes, train=False, seed=3)
    x = X[:1].contiguous()
    eager = _timed(lambda: one.forward(x), 100)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        one.forward(x)
    print(f"one token: {eager * 1e3:.1f} us, as a graph {_timed(graph.replay, 100) * 1e3:.1f} us")


if __name__ == "__main__":
    main()
