"""The grouped router, rows in 8 bits and their products in 64 bits, from their definitions.  Every function takes CPU tensors;
tolerances are those of moe_reference.py (one rounding to the type, 2^-24 of the terms for each of a few float32 roundings)."""
import math

import torch

import moe_reference as ref

BLOCK = 32


# ------------------------------------------------------------------------------------------------ router
def scores_of(logits, scores):
    """(scores that choices are made by, without the NaN; scores that weights are made of)"""
    l = logits.double()
    if scores == "sigmoid":
        s = 1.0 / (1.0 + torch.exp(-l))
        return s, s
    clean = torch.where(torch.isnan(l), -math.inf, l)
    most = clean.amax(1, keepdim=True)
    e = torch.where(clean == most, 1.0, torch.exp(clean - most))
    return e / e.sum(1, keepdim=True), torch.exp(l - l.amax(1, keepdim=True)) / torch.exp(l - l.amax(1, keepdim=True)).sum(1, keepdim=True)


def route(logits, k, scores, bias, n_groups, top_groups, group_top, normalise, scale):
    """(experts, weights): token by token, group by group."""
    T, E = logits.shape
    each = E // n_groups
    by, s = scores_of(logits, scores)
    c = by if bias is None else by + bias.double()
    alive = (logits > -math.inf) & (c > -math.inf)
    experts = torch.full((T, k), -1, dtype=torch.int32)
    weights = torch.zeros(T, k, dtype=torch.float64)
    for t in range(T):
        keys = [float(c[t, e]) if alive[t, e] else None for e in range(E)]
        of_group = []
        for g in range(n_groups):
            best = sorted((v for v in keys[g * each:(g + 1) * each] if v is not None), reverse=True)[:group_top]
            of_group.append((sum(best), -g) if best else None)
        kept = sorted((g for g in of_group if g is not None), reverse=True)[:top_groups]
        groups = {-g for _, g in kept}
        left = sorted(((-keys[e], e) for e in range(E) if keys[e] is not None and e // each in groups))[:k]
        chosen = [e for _, e in left]
        if not chosen:
            continue
        at = torch.tensor(chosen)
        experts[t, :len(chosen)] = at.to(torch.int32)
        l = logits[t, at].double()
        if not normalise:
            w = s[t, at]
        elif scores == "sigmoid":
            w = torch.softmax(torch.nn.functional.logsigmoid(l), 0)
        else:
            w = torch.softmax(l, 0)
        weights[t, :len(chosen)] = scale * w
    return experts, weights


def route_gradient(logits, experts, d_weights, scores, normalise, scale):
    l = torch.where(torch.isinf(logits.double()), -1e300, logits.double()).requires_grad_()
    live = experts >= 0
    log_s = torch.nn.functional.logsigmoid(l) if scores == "sigmoid" else torch.log_softmax(l, 1)
    picked = torch.gather(log_s, 1, experts.long().clamp(min=0))
    if normalise:
        picked = torch.log_softmax(torch.where(live, picked, -1e300), 1)
    w = torch.where(live, scale * torch.exp(picked), 0.0)
    grad, = torch.autograd.grad((w * torch.where(live, d_weights.double(), 0.0)).sum(), l)
    return torch.where(live.any(1, keepdim=True), grad, 0.0)


# ------------------------------------------------------------------------------------------------ 8 bits
def to_even(v):
    low = torch.floor(v)
    up = (v - low > 0.5) | ((v - low == 0.5) & (low % 2 != 0))
    return low + up


def quantise(X):
    """(codes int8, scales float32).  A quotient of two float32 numbers that is not half a whole number is at least 2^-33 from it, which
    64 bits tell."""
    x = X.double()
    most = x.abs().amax(1) if X.shape[1] else torch.zeros(X.shape[0], dtype=torch.float64)
    bad = ~torch.isfinite(most)
    scales = torch.where(bad, math.nan, most.float() / torch.tensor(127.0))
    s = scales.double()
    usable = ~bad & (s > 0)
    q = to_even(torch.where(usable[:, None], x, 0.0) / torch.where(usable, s, 1.0)[:, None]).clamp(-127, 127)
    return q.to(torch.int8), scales


def pack(X):
    """(codes int8, exponents uint8)"""
    n, w = X.shape
    least = -24 if X.dtype is torch.float16 else -126
    powers = torch.arange(least, 128)
    borders = 127.5 * torch.exp2(powers.double())
    codes, exponents = torch.zeros(n, w, dtype=torch.int8), torch.zeros(n, -(-w // BLOCK), dtype=torch.uint8)
    for b in range(exponents.shape[1]):
        part = X[:, b * BLOCK:(b + 1) * BLOCK].double()
        most = part.abs().amax(1)
        bad = ~torch.isfinite(most)
        which = torch.searchsorted(borders, torch.where(bad, 0.0, most), right=True)
        unit = torch.exp2(powers[which].double())[:, None]
        q = to_even(torch.where(bad[:, None], 0.0, part) / unit)
        q = torch.where((q * unit).abs() > torch.finfo(X.dtype).max, 63.0 * torch.sign(q), q)
        codes[:, b * BLOCK:(b + 1) * BLOCK] = q.to(torch.int8)
        exponents[:, b] = torch.where(bad, 255, powers[which] + 127).to(torch.uint8)
    return codes, exponents


def kept(codes, exponents, dtype):
    """What the codes stand for, as the type (exactly, or this fails)."""
    e = exponents.long().repeat_interleave(BLOCK, 1)[:, :codes.shape[1]]
    v = torch.where(e == 255, math.nan, codes.double() * torch.exp2(e.double() - 127))
    out = v.to(dtype)
    same = (out.double() == v) | torch.isnan(v)
    assert same.all()
    return out


def unpacked(values, name):
    """(act(values), its bound)"""
    z = values.double()
    y = ref.activation(z, name)
    if name == "none":
        return y, torch.zeros_like(y)
    if name == "swiglu":
        g, u = z.chunk(2, dim=1)
        terms = 1.2 * g.abs() * u.abs()
    else:
        terms = 1.2 * z.abs()
    return y, ref.bound(y, terms, 1, values.dtype)


def product(parts, rows, X, x_scales, W, w_scales, bias, residual, name, dtype):
    """(y, its bound, z, its bound): whole sums, then a few float32 roundings."""
    wide = W.shape[1]
    z = torch.zeros(rows, wide, dtype=torch.float64)
    size = torch.zeros_like(z)
    d_out = wide // 2 if name == "swiglu" else wide
    r = torch.zeros(rows, d_out, dtype=torch.float64)
    for e, s, x in parts:
        z[s] = (X[x].double() @ W[e].double().t()) * x_scales[x].double()[:, None] * w_scales[e].double()
        size[s] = z[s].abs()
        if bias is not None:
            z[s] += bias[e].double()
            size[s] += bias[e].double().abs()
        if residual is not None:
            r[s] = residual[s].double()
    act = ref.activation(z, name)
    if name == "swiglu":
        g, u = z.chunk(2, dim=1)
        sg, su = size.chunk(2, dim=1)
        terms = 1.2 * sg * u.abs() + ref.activation(g, "silu").abs() * su + act.abs() + sg * su * 2.0 ** -18
    else:
        terms = 1.2 * size
    y = act + r
    return y, ref.bound(y, terms + r.abs(), 1, dtype), z, ref.bound(z, size, 1, dtype)
