"""The operators of a mixture-of-experts layer in 64 bits, from their definitions, with the error that a result may have.

Every function takes CPU tensors and returns float64 results and, where the result is a rounded sum, a bound on the error:
UNIT[type] * |result| for the one rounding to the type, and for the float32 arithmetic before it 2^-24 times the sum of the
terms' magnitudes times 4 * (sqrt(n) + 8) for n terms in any order (a random walk of n roundings, and a few for the
activation), times 1.2 for the steepest slope of an activation (gelu's and silu's are below 1.13)."""
import math

import torch

UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -126}  # (float16 has its subnormals)


def bound(value, terms, n, dtype):
    return 1.01 * UNIT[dtype] * value.abs() + 4.0 * (math.sqrt(n) + 8.0) * 2.0 ** -24 * terms + TINY[dtype]


def check(got, want, limit, what):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, f"{what}: shape {list(got.shape)}, expected {list(want.shape)}"
    both = torch.isnan(want)
    assert torch.equal(torch.isnan(got), both), f"{what}: NaN in {int((torch.isnan(got) != both).sum())} other places"
    over = torch.where(both, 0.0, (got - want).abs() - limit)
    assert got.numel() == 0 or float(over.max()) <= 0.0, \
        f"{what}: off by {float((got - want).abs()[over > 0].max()):.3e} in {int((over > 0).sum())} of {over.numel()} places"


def route(logits, k, normalise):
    """(experts, weights)"""
    l = logits.double()
    T, E = l.shape
    key = torch.where(torch.isnan(l), -math.inf, l)
    order = torch.argsort(key, dim=1, descending=True, stable=True)[:, :k]
    top = torch.gather(key, 1, order)
    experts = torch.where(top > -math.inf, order, -1)
    picked = torch.where(experts >= 0, top, -math.inf)
    inside = picked if normalise else l
    # (the largest is taken off first: log of the sum would be lost beside logits of the type's lowest value)
    most = inside.amax(1, keepdim=True)
    weights = torch.exp(picked - most) / torch.exp(inside - most).sum(1, keepdim=True)
    weights = torch.where(experts >= 0, weights, 0.0)
    return experts.to(torch.int32), weights


def route_gradient(logits, experts, d_weights, normalise):
    l = torch.where(torch.isinf(logits.double()), -1e300, logits.double()).requires_grad_()
    live = experts >= 0
    if normalise:
        picked = torch.where(live, torch.gather(l, 1, experts.long().clamp(min=0)), -1e300)
        w = torch.softmax(picked, 1)
    else:
        w = torch.gather(torch.softmax(l, 1), 1, experts.long().clamp(min=0))
    total = torch.where(live, w * torch.where(live, d_weights.double(), 0.0), 0.0).sum()
    grad, = torch.autograd.grad(total, l)
    return torch.where(live.any(1, keepdim=True), grad, 0.0)


def sort(experts, E):
    """(expert_ptr, entry_of, slot_of)"""
    flat = experts.reshape(-1).tolist()
    lists = [[] for _ in range(E)]
    for i, e in enumerate(flat):
        if 0 <= e < E:
            lists[e].append(i)
    ptr, entry, slot = [0], [], [-1] * len(flat)
    for one in lists:
        for i in one:
            slot[i] = len(entry)
            entry.append(i)
        ptr.append(len(entry))
    entry += [-1] * (len(flat) - len(entry))
    return [torch.tensor(v, dtype=torch.int32) for v in (ptr, entry, slot)]


def activation(z, name):
    if name == "relu":
        return torch.relu(z)
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z / math.sqrt(2.0)))
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "swiglu":
        g, u = z.chunk(2, dim=1)
        return g * torch.sigmoid(g) * u
    return z


def slope(d, z, name):
    """d times the derivative at z, by autograd."""
    at = z.detach().clone().requires_grad_()
    grad, = torch.autograd.grad(activation(at, name), at, d)
    return grad


def groups(order, k, E, rows, gather):
    """(expert, its sorted rows, the rows of X they take)"""
    if order is None:
        return [(0, torch.arange(rows), torch.arange(rows))]
    ptr, entry, _ = order
    out = []
    for e in range(E):
        s = torch.arange(int(ptr[e]), int(ptr[e + 1]))
        out.append((e, s, entry[s].long() // k if gather else s))
    return out


def product(parts, rows, X, W, bias, residual, name):
    """(y, its bound, z, its bound)"""
    dtype, wide, d_in = X.dtype, W.shape[1], W.shape[2]
    z = torch.zeros(rows, wide, dtype=torch.float64)
    size = torch.zeros_like(z)
    d_out = wide // 2 if name == "swiglu" else wide
    r = torch.zeros(rows, d_out, dtype=torch.float64)
    for e, s, x in parts:
        a, w = X[x].double(), W[e].double()
        z[s], size[s] = a @ w.t(), a.abs() @ w.abs().t()
        if bias is not None:
            z[s] += bias[e].double()
            size[s] += bias[e].double().abs()
        if residual is not None:
            r[s] = residual[s].double()
    act = activation(z, name)
    if name == "swiglu":
        g, u = z.chunk(2, dim=1)
        sg, su = size.chunk(2, dim=1)
        terms = 1.2 * sg * u.abs() + activation(g, "silu").abs() * su + act.abs()
        # (the product of both errors)
        terms = terms + sg * su * 4.0 * (math.sqrt(d_in) + 8.0) * 2.0 ** -24
    else:
        terms = 1.2 * size
    y = act + r
    return y, bound(y, terms + r.abs(), d_in, dtype), z, bound(z, size, d_in, dtype)


def product_dx(parts, rows, dZ, W, pre, name):
    d = torch.zeros(rows, W.shape[2], dtype=torch.float64)
    size = torch.zeros_like(d)
    for e, s, _ in parts:
        d[s], size[s] = dZ[s].double() @ W[e].double(), dZ[s].double().abs() @ W[e].double().abs()
    if name == "none":
        return d, bound(d, size, W.shape[1], dZ.dtype)
    z = torch.zeros_like(pre, dtype=torch.float64)
    for _, s, _ in parts:
        z[s] = pre[s].double()
    if name == "swiglu":
        g, u = z.chunk(2, dim=1)
        # (the slope's own sum 1 + z (1 - s) may cancel: its terms)
        terms = torch.cat([size * u.abs() * (1.2 + g.abs()), size * (1.0 + g.abs())], 1)
    else:
        terms = size * (1.2 + z.abs())
    out = slope(d, z, name)
    return out, bound(out, terms, W.shape[1], dZ.dtype)


def product_dw(parts, dZ, X, E):
    dW = torch.zeros(E, dZ.shape[1], X.shape[1], dtype=torch.float64)
    size = torch.zeros_like(dW)
    db = torch.zeros(E, dZ.shape[1], dtype=torch.float64)
    db_size = torch.zeros_like(db)
    n = 1
    for e, s, x in parts:
        dz, a = dZ[s].double(), X[x].double()
        dW[e], size[e] = dz.t() @ a, dz.abs().t() @ a.abs()
        db[e], db_size[e] = dz.sum(0), dz.abs().sum(0)
        n = max(n, len(s))
    return dW, bound(dW, size, n, dZ.dtype), db, bound(db, db_size, n, dZ.dtype)
