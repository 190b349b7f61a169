"""More operators of a mixture-of-experts layer, as measurable cases.

`route`: a router whose scores are a softmax or sigmoids, with a bias that balances the experts' load, groups of experts of
which a token may use some, and the weights renormalised; and its gradient.  `int8`: the rows of a batch brought to 8-bit integers
with a scale each, and every expert's product of them with weights of 8-bit integers with a scale for each output channel.
`rows8`: activations kept as checkpoints of 8 bits and read back, with the activation that follows them.  `backward8`: the
gradients of an expert's two products that use such checkpoints: of the inputs, through the derivative of the activation at a
kept z, and of the weights, with a kept x.

T tokens choose k of E experts each; entry t * k + j is token t's choice j.  An entry whose expert is outside 0 .. E - 1 is
dropped.  Sorted rows are in the order of the experts, inside an expert in the order of the entries; rows past the last
kept entry are zero.
"""
from __future__ import annotations

import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}
_BLOCK = 32  # columns of a checkpoint's row that share an exponent


def _route(name, tokens, experts, top_k, dtype, scores, groups, top_groups, group_top, bias, normalise, scale, masked, train):
    """group_top: how many of a group's largest make its score.  masked: share of the tokens that are padding (all their logits
    -inf); of the others' logits a tenth of it, too."""
    return {"name": name, "op": "route", "tokens": tokens, "experts": experts, "top_k": top_k, "dtype": dtype, "scores": scores,
            "groups": groups, "top_groups": top_groups, "group_top": group_top, "bias": bias, "normalise": normalise,
            "scale": scale, "masked": masked, "train": train}


def _int8(name, tokens, experts, top_k, d_in, d_out, dtype, activation, bias, residual, dropped):
    """experts 0: no routing, one dense product.  dtype: of X, Y, bias and residual."""
    return {"name": name, "op": "int8", "tokens": tokens, "experts": experts, "top_k": top_k, "d_in": d_in, "d_out": d_out,
            "dtype": dtype, "activation": activation, "bias": bias, "residual": residual, "dropped": dropped}


def _rows8(name, rows, width, dtype, activation):
    return {"name": name, "op": "rows8", "rows": rows, "width": width, "dtype": dtype, "activation": activation}


def _backward8(name, tokens, experts, top_k, width, hidden, dtype, activation, dropped):
    """A layer of tokens of `width`, with `hidden` activations between an expert's two products."""
    return {"name": name, "op": "backward8", "tokens": tokens, "experts": experts, "top_k": top_k, "width": width,
            "hidden": hidden, "dtype": dtype, "activation": activation, "dropped": dropped}


def listed():
    return [
        # one token of one user's answer: nothing but latency
        _route("route_token", 1, 256, 8, "bf16", "sigmoid", 8, 4, 2, True, True, 2.5, 0.0, False),
        # a training batch of many small experts with its gradient
        _route("route_batch", 16384, 256, 8, "f32", "sigmoid", 8, 4, 2, True, True, 2.5, 0.0, True),
        # a ragged batch with padding tokens and experts that are switched off, softmax scores, groups by their best expert
        _route("route_ragged", 5003, 60, 6, "f16", "softmax", 6, 3, 1, False, False, 1.0, 0.07, True),
        # one token's experts: the weights are read once, eight rows are computed
        _int8("int8_token", 1, 64, 8, 2048, 1024, "bf16", "swiglu", False, False, 0.0),
        # the tokens of a batch of users, a dozen rows an expert
        _int8("int8_users", 96, 32, 4, 1024, 2048, "f16", "silu", True, False, 0.0),
        # a prompt through eight large gated experts: the largest product
        _int8("int8_prompt", 8192, 8, 2, 2048, 4096, "bf16", "swiglu", False, False, 0.0),
        # an ordinary dense layer
        _int8("int8_dense", 8192, 0, 1, 4096, 4096, "f16", "gelu", True, True, 0.0),
        # odd sizes, dropped entries, results in single precision
        _int8("int8_odd", 2003, 10, 2, 1000, 777, "f32", "relu", True, True, 0.05),
        # what a gated layer's first product made, kept and read back as what its second one takes
        _rows8("rows8_train", 16384, 4096, "bf16", "swiglu"),
        # odd rows of single precision, kept and read back as they are
        _rows8("rows8_odd", 3001, 1111, "f32", "none"),
        # the gradients of a training step of 32 gated experts
        _backward8("backward8_train", 8192, 32, 4, 1024, 1024, "bf16", "swiglu", 0.0),
        # odd sizes, dropped entries
        _backward8("backward8_odd", 2003, 10, 2, 1000, 777, "f16", "gelu", 0.05),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Mostly whole tiles, some whole 16-byte words, some odd."""
    n, kind = _log_int(rng, lo, hi), rng.random()
    return max(64, (n + 32) // 64 * 64) if kind < 0.6 else max(8, n // 8 * 8) if kind < 0.8 else n | 1


def draw(rng):
    op = rng.choice(("route", "int8", "int8", "rows8", "backward8"))
    tokens = _log_int(rng, 1, 16384)
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    experts = _log_int(rng, 2, 128)
    top_k = rng.randint(1, min(8, experts))
    activation = rng.choice(("none", "relu", "gelu", "silu", "swiglu", "swiglu"))
    if op == "route":
        groups = rng.choice((1, 1, 2, 4, 6, 8))
        each = _log_int(rng, 2, 256 // groups)
        experts, top_groups = groups * each, rng.randint(1, groups)
        case = _route("", tokens, experts, rng.randint(1, min(8, top_groups * each)), dtype, rng.choice(("sigmoid", "softmax")),
                      groups, top_groups, rng.choice((1, 2)), rng.random() < 0.7, rng.random() < 0.6, rng.choice((1.0, 2.5)),
                      rng.choice((0.0, 0.0, 0.07)), rng.random() < 0.5)
    elif op == "int8":
        if rng.random() < 0.15:
            experts, top_k = 0, 1
        d_in, d_out = _width(rng, 64, 4096), _width(rng, 64, 4096)
        if experts:
            experts = max(top_k, min(experts, 300000000 // (d_in * d_out)))
        most = 4.0e11 / (2.0 if activation == "swiglu" else 1.0)
        tokens = max(1, min(tokens, int(most / (2.0 * top_k * d_in * d_out))))
        case = _int8("", tokens, experts, top_k, d_in, d_out, dtype, activation, rng.random() < 0.5, rng.random() < 0.3,
                     rng.choice((0.0, 0.0, 0.1)) if experts else 0.0)
    elif op == "rows8":
        width = _width(rng, 64, 4096)
        if activation == "swiglu":
            width += width % 2
        case = _rows8("", max(1, min(4 * tokens, 67000000 // width)), width, dtype, activation)
    else:
        width, hidden = _width(rng, 64, 4096), _width(rng, 64, 4096)
        if activation == "none":
            activation = "gelu"  # (there is always one between the two products)
        experts = max(top_k, min(experts, 100000000 // (width * hidden)))
        most = (6.0e10 if dtype == "f32" else 4.0e11) / (3.0 if activation == "swiglu" else 2.0)
        tokens = max(1, min(tokens, int(most / (2.0 * top_k * width * hidden))))
        case = _backward8("", tokens, experts, top_k, width, hidden, dtype, activation, rng.choice((0.0, 0.0, 0.1)))
    del case["name"]
    return case


# ----------------------------------------------------------------------------------------------------- inputs
def _popular(T, E, gen):
    """Router logits: some experts are chosen several times as often as others."""
    popularity = -0.5 * torch.log(1.0 + torch.randperm(E, generator=gen, device="cuda").float())
    return popularity + 1.5 * torch.randn(T, E, generator=gen, device="cuda")


def _choices(case, gen):
    """int32 [T, k]: distinct experts of every token, an exact number of entries dropped at random (-1)."""
    T, E, k = case["tokens"], case["experts"], case["top_k"]
    chosen = torch.argsort(_popular(T, E, gen), dim=1, descending=True)[:, :k].contiguous().to(torch.int32)
    n = int(round(case["dropped"] * T * k))
    if n:
        chosen.view(-1)[torch.randperm(T * k, generator=gen, device="cuda")[:n]] = -1
    return chosen


def _wide(n, activation):
    return 2 * n if activation == "swiglu" else n


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 1000003 + 29)
    dtype = _TYPES[case["dtype"]]

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dtype)

    def empty(*shape, dtype=dtype):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    s = {"case": case}
    if case["op"] == "route":
        T, E, k = case["tokens"], case["experts"], case["top_k"]
        logits = _popular(T, E, gen)
        # the bias that balances such scores: against the more popular experts
        s["bias"] = 0.1 * torch.randn(E, generator=gen, device="cuda") if case["bias"] else None
        if case["masked"]:
            logits[torch.rand(T, E, generator=gen, device="cuda") < case["masked"] / 10] = -math.inf
            logits[torch.rand(T, generator=gen, device="cuda") < case["masked"]] = -math.inf
        s["logits"] = logits.to(dtype)
        s["d_weights"] = torch.randn(T, k, generator=gen, device="cuda")
        if own:
            s["experts"], s["weights"] = empty(T, k, dtype=torch.int32), empty(T, k, dtype=torch.float32)
            s["d_logits"] = torch.empty_like(s["logits"])
    elif case["op"] == "int8":
        T, E, k, K, N = case["tokens"], case["experts"], case["top_k"], case["d_in"], case["d_out"]
        rows, wide = T * k, _wide(N, case["activation"])
        if E:
            s["experts"] = _choices(case, gen)
        # (a few columns of activations are several times as large as the others)
        s["X"] = (normal(T, K).float() * torch.exp(0.5 * torch.randn(K, generator=gen, device="cuda"))).to(dtype)
        W = torch.randn(max(E, 1), wide, K, generator=gen, device="cuda") * K ** -0.5
        s["W_scales"] = W.abs().amax(2) / 127.0
        s["W"] = torch.round(W / s["W_scales"][:, :, None]).to(torch.int8)
        s["bias"] = normal(max(E, 1), wide, scale=0.5) if case["bias"] else None
        s["residual"] = normal(rows, N) if case["residual"] else None
        if own:
            s["Xq"], s["X_scales"], s["Y_out"] = empty(T, K, dtype=torch.int8), empty(T, dtype=torch.float32), empty(rows, N)
    elif case["op"] == "rows8":
        n, w = case["rows"], case["width"]
        # (rows of different sizes, as tokens have)
        s["X"] = (normal(n, w).float() * torch.exp(torch.randn(n, 1, generator=gen, device="cuda"))).to(dtype)
        if own:
            s["codes"], s["exponents"] = empty(n, w, dtype=torch.int8), empty(n, -(-w // _BLOCK), dtype=torch.uint8)
            s["Y_out"] = empty(n, w // 2 if case["activation"] == "swiglu" else w)
    else:
        T, E, k, D, H = case["tokens"], case["experts"], case["top_k"], case["width"], case["hidden"]
        rows, wide = T * k, _wide(H, case["activation"])
        s["experts"] = _choices(case, gen)
        s["X"], s["pre"] = normal(T, D), normal(rows, wide)
        s["W2"] = normal(E, D, H, scale=H ** -0.5)
        # of the second product's results and of the first one's
        s["d_ys"], s["d_z"] = normal(rows, D), normal(rows, wide)
        if own:
            s["X8"], s["X_exponents"] = empty(T, D, dtype=torch.int8), empty(T, -(-D // _BLOCK), dtype=torch.uint8)
            s["pre8"], s["pre_exponents"] = empty(rows, wide, dtype=torch.int8), empty(rows, -(-wide // _BLOCK), dtype=torch.uint8)
            s["d_pre_out"] = empty(rows, wide)
            s["dW1_out"], s["db1_out"] = empty(E, wide, D), empty(E, wide)
    if "experts" in s and case["op"] != "route":
        # a program sorts once for every operator that uses the order
        s["order"] = _sorted(s["experts"], case["experts"])
        s["bounds"] = s["order"][0].tolist()
        if own:
            import paper_2207_04606_amd as sptir
            s["routing"] = sptir.sptir_moe_sort(s["experts"], case["experts"])
    return s


# ----------------------------------------------------------------------------------------------------- the plain forms
def _sorted(experts, E):
    """(expert_ptr [E + 1], entry_of [N], slot_of [N]), all int32."""
    flat = experts.reshape(-1).long()
    group = torch.where((flat >= 0) & (flat < E), flat, E)
    order = torch.argsort(group, stable=True)
    ptr = torch.searchsorted(group[order], torch.arange(E + 1, device=flat.device))
    slot = torch.empty_like(order)
    slot[order] = torch.arange(order.numel(), device=flat.device)
    kept = group[order] < E
    return (ptr.to(torch.int32), torch.where(kept, order, -1).to(torch.int32),
            torch.where(group < E, slot, -1).to(torch.int32))


def _plain_scores(l, scores):
    """(scores, their logarithms) in 64 bits: two of them may be closer than 32 bits tell."""
    if scores == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-l)), torch.clamp(l, max=0.0) - torch.log1p(torch.exp(-l.abs()))
    most = l.amax(1, keepdim=True)
    most = torch.where(most > -math.inf, most, 0.0)
    e = torch.exp(l - most)
    total = e.sum(1, keepdim=True)
    total = torch.where(total > 0.0, total, 1.0)
    return e / total, l - most - torch.log(total)


def _plain_route(s):
    case, l = s["case"], s["logits"].double()
    T, E = l.shape
    k, G, normalise = case["top_k"], case["groups"], case["normalise"]
    score, log_score = _plain_scores(l, case["scores"])
    c = score if s["bias"] is None else score + s["bias"].double()
    c = torch.where(l > -math.inf, c, -math.inf)
    if case["top_groups"] < G:
        best = torch.sort(c.view(T, G, E // G), dim=2, descending=True)[0][:, :, :case["group_top"]]
        of_group = torch.where(best > -math.inf, best, 0.0).sum(2)
        of_group = torch.where(best[:, :, 0] > -math.inf, of_group, -math.inf)
        kept = torch.sort(of_group, dim=1, descending=True, stable=True)[1][:, :case["top_groups"]]
        inside = torch.zeros(T, G, dtype=torch.bool, device=l.device).scatter_(1, kept, True)
        c = torch.where(inside.repeat_interleave(E // G, 1), c, -math.inf)
    top, chosen = torch.sort(c, dim=1, descending=True, stable=True)
    top, chosen = top[:, :k], chosen[:, :k]
    valid = top > -math.inf
    picked = torch.where(valid, torch.gather(log_score, 1, chosen), -math.inf)
    if normalise:
        most = picked.amax(1, keepdim=True)
        p = torch.exp(picked - torch.where(most > -math.inf, most, 0.0))
        total = p.sum(1, keepdim=True)
        p = p / torch.where(total > 0.0, total, 1.0)
    else:
        p = torch.exp(picked)
    out = [torch.where(valid, chosen, -1).to(torch.int32), (case["scale"] * p).float()]
    if case["train"]:
        dw = case["scale"] * torch.where(valid, s["d_weights"].double(), 0.0)
        mean = (p * dw).sum(1, keepdim=True)
        if case["scores"] == "sigmoid":
            falls = 1.0 - torch.gather(score, 1, chosen)
            of_choice = p * falls * (dw - mean if normalise else dw)
            d = torch.zeros_like(l).scatter_add_(1, chosen, torch.where(valid, of_choice, 0.0))
        elif normalise:
            d = torch.zeros_like(l).scatter_add_(1, chosen, torch.where(valid, p * (dw - mean), 0.0))
        else:
            d = torch.zeros_like(l).scatter_add_(1, chosen, torch.where(valid, p * dw, 0.0)) - score * mean
        out.append(d.to(s["logits"].dtype))
    return out


def _plain_activation(z, name):
    if name == "relu":
        return torch.where(z > 0, z, 0.0)
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    if name == "swiglu":
        g, u = z.chunk(2, dim=-1)
        return g / (1.0 + torch.exp(-g)) * u
    return z


def _plain_slope(d, z, name):
    """d times the derivative of the activation at z."""
    if name == "relu":
        return torch.where(z > 0, d, 0.0)
    if name == "gelu":
        return d * (0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (0.5 / math.pi) ** 0.5)
    if name == "silu":
        g = 1.0 / (1.0 + torch.exp(-z))
        return d * g * (1.0 + z * (1.0 - g))
    if name == "swiglu":
        a, u = z.chunk(2, dim=-1)
        g = 1.0 / (1.0 + torch.exp(-a))
        return torch.cat([d * u * g * (1.0 + a * (1.0 - g)), d * a * g], dim=-1)
    return d


def _groups(s):
    case = s["case"]
    if not case["experts"]:
        return [(0, 0, case["tokens"])]
    b = s["bounds"]
    return [(e, b[e], b[e + 1]) for e in range(case["experts"]) if b[e + 1] > b[e]]


def _plain_int8(s):
    case, X, W = s["case"], s["X"].float(), s["W"]
    rows, N, K, dtype = case["tokens"] * case["top_k"], case["d_out"], case["d_in"], s["X"].dtype
    # (by a tensor: by a number torch multiplies with its reciprocal)
    scale = X.abs().amax(1) / torch.full((), 127.0, device=X.device)
    # (64 bits: a quotient next to the middle between two integers)
    q = torch.round(X.double() / torch.where(scale > 0.0, scale, 1.0).double()[:, None]).clamp(-127.0, 127.0).float()
    token = s["order"][1].long() // case["top_k"] if case["experts"] else None
    Y = torch.zeros(rows, N, dtype=dtype, device=X.device)
    for e, lo, hi in _groups(s):
        at = slice(lo, hi) if token is None else token[lo:hi]
        x, w = q[at], W[e].float()
        # (whole numbers: 1024 products of 127 * 127 stay below 2^24)
        z = torch.zeros(hi - lo, W.shape[1], dtype=torch.float64, device=X.device)
        for c in range(0, K, 1024):
            z += x[:, c:c + 1024] @ w[:, c:c + 1024].t()
        z = z.float() * scale[at][:, None] * s["W_scales"][e]
        if s["bias"] is not None:
            z = z + s["bias"][e].float()
        y = _plain_activation(z, case["activation"])
        if s["residual"] is not None:
            y = y + s["residual"][lo:hi].float()
        Y[lo:hi] = y.to(dtype)
    return [scale, Y]


def _plain_kept(X):
    """(what a checkpoint holds of the rows, its exponents plus 127)"""
    n, w = X.shape
    dtype, least = X.dtype, -24 if X.dtype is torch.float16 else -126
    blocks = -(-w // _BLOCK)
    v = torch.zeros(n, blocks * _BLOCK, device=X.device)
    v[:, :w] = X.float()
    v = v.view(n, blocks, _BLOCK)
    most = v.abs().amax(2)
    mantissa, e = torch.frexp(most)  # (mantissa in [1/2, 1))
    e = e - torch.where(mantissa < 255.0 / 256.0, 7, 6)
    e = torch.where(most > 0.0, e, least).clamp(min=least)
    q = torch.round(torch.ldexp(v, -e[:, :, None]))
    kept = torch.ldexp(q, e[:, :, None])
    # (64 at the topmost exponent is past the type's range)
    kept = torch.where(kept.abs() > torch.finfo(dtype).max, torch.ldexp(torch.sign(q) * 63.0, e[:, :, None]), kept)
    return kept.view(n, -1)[:, :w], (e + 127).to(torch.uint8)


def _plain_rows8(s):
    kept, exponents = _plain_kept(s["X"])
    return [exponents, _plain_activation(kept, s["case"]["activation"]).to(s["X"].dtype)]


def _plain_backward8(s):
    case, dtype = s["case"], s["X"].dtype
    rows, D, wide = case["tokens"] * case["top_k"], case["width"], s["pre"].shape[1]
    (X, _), (pre, _) = _plain_kept(s["X"]), _plain_kept(s["pre"])
    token = s["order"][1].long() // case["top_k"]
    d_pre = torch.zeros(rows, wide, dtype=dtype, device=X.device)
    dW = torch.zeros(case["experts"], wide, D, dtype=dtype, device=X.device)
    db = torch.zeros(case["experts"], wide, dtype=dtype, device=X.device)
    for e, lo, hi in _groups(s):
        d = s["d_ys"][lo:hi].float() @ s["W2"][e].float()
        d_pre[lo:hi] = _plain_slope(d, pre[lo:hi], case["activation"]).to(dtype)
        dz = s["d_z"][lo:hi].float()
        dW[e] = (dz.t() @ X[token[lo:hi]]).to(dtype)
        db[e] = dz.sum(0).to(dtype)
    return [d_pre, dW, db]


# ----------------------------------------------------------------------------------------------------- the framework's
def _own_route(s):
    import paper_2207_04606_amd as sptir
    case = s["case"]
    how = {"scores": case["scores"], "bias": s["bias"], "n_groups": case["groups"], "top_groups": case["top_groups"],
           "group_top": case["group_top"], "normalise": case["normalise"], "scale": case["scale"]}
    sptir.sptir_moe_route_groups(s["logits"], s["experts"], s["weights"], **how)
    out = [s["experts"], s["weights"]]
    if case["train"]:
        sptir.sptir_moe_route_groups_backward(s["logits"], s["experts"], s["weights"], s["d_weights"], s["d_logits"],
                                              scores=case["scores"], normalise=case["normalise"], scale=case["scale"])
        out.append(s["d_logits"])
    return out


def _own_int8(s):
    import paper_2207_04606_amd as sptir
    case = s["case"]
    sptir.sptir_moe_quantise(s["X"], s["Xq"], s["X_scales"])
    sptir.sptir_moe_product_int8(s.get("routing"), s["Xq"], s["X_scales"], s["W"], s["W_scales"], s["Y_out"], bias=s["bias"],
                                 residual=s["residual"], activation=case["activation"], gather=bool(case["experts"]))
    return [s["X_scales"], s["Y_out"]]


def _own_rows8(s):
    import paper_2207_04606_amd as sptir
    sptir.sptir_moe_pack(s["X"], s["codes"], s["exponents"])
    sptir.sptir_moe_unpack(s["codes"], s["exponents"], s["Y_out"], activation=s["case"]["activation"])
    return [s["exponents"], s["Y_out"]]


def _own_backward8(s):
    import paper_2207_04606_amd as sptir
    case, r = s["case"], s["routing"]
    sptir.sptir_moe_pack(s["X"], s["X8"], s["X_exponents"])
    sptir.sptir_moe_pack(s["pre"], s["pre8"], s["pre_exponents"])
    sptir.sptir_moe_product_dx_packed(r, s["d_ys"], s["W2"], s["d_pre_out"], s["pre8"], s["pre_exponents"],
                                      activation=case["activation"])
    sptir.sptir_moe_product_dw_packed(r, s["d_z"], s["X8"], s["X_exponents"], s["dW1_out"], db=s["db1_out"], gather=True)
    return [s["d_pre_out"], s["dW1_out"], s["db1_out"]]


def run(state):
    op = state["case"]["op"]
    if own:
        return {"route": _own_route, "int8": _own_int8, "rows8": _own_rows8, "backward8": _own_backward8}[op](state)
    return {"route": _plain_route, "int8": _plain_int8, "rows8": _plain_rows8, "backward8": _plain_backward8}[op](state)


# ----------------------------------------------------------------------------------------------------- costs
def work(case):
    b = _BYTES[case["dtype"]]
    if case["op"] == "rows8":
        # the rows, the checkpoint there and back, what is made of it
        n, w = case["rows"], case["width"]
        size = n * w * (b + 2.0 + 2.0 / _BLOCK) + n * (w // 2 if case["activation"] == "swiglu" else w) * b
        return {"bytes": float(size), "flops": 4.0 * n * w}
    T, E, k = case["tokens"], case["experts"], case["top_k"]
    n = T * k
    if case["op"] == "route":
        # the logits; ids and weights; with the gradient the weights' gradient and the logits'
        size, flops = T * E * b + n * 8 + (E * 4 if case["bias"] else 0), 6.0 * T * E
        if case["train"]:
            size += n * 4 + T * E * b
            flops += 4.0 * T * E
        return {"bytes": float(size), "flops": flops}
    kept = n - int(round(case["dropped"] * n))
    used = E * (1.0 - (1.0 - k / E) ** T) if E else 1.0
    if case["op"] == "int8":
        K, N = case["d_in"], case["d_out"]
        wide = _wide(N, case["activation"])
        size = T * K * b + T * 4 + used * wide * (K + 4) + n * N * b
        size += (kept * N * b if case["residual"] else 0) + (used * wide * b if case["bias"] else 0)
        return {"bytes": float(size), "flops": 2.0 * kept * K * wide}
    D, H = case["width"], case["hidden"]
    wide = _wide(H, case["activation"])
    # x and z into their checkpoints and from there, two gradients, the weights, and three results
    size = (T * D + n * wide) * (b + 2.0 + 2.0 / _BLOCK) + (n * D + n * wide) * b + used * D * H * b + (n * wide + E * wide * (D + 1)) * b
    return {"bytes": float(size), "flops": 2.0 * kept * D * (H + wide)}


# ----------------------------------------------------------------------------------------------------- in 64 bits
def _exact_route(s):
    case, l = s["case"], s["logits"].double()
    T, E = l.shape
    k, G = case["top_k"], case["groups"]
    f = torch.nn.functional
    dead = l == -math.inf
    at = torch.where(dead, -1e300, l).requires_grad_()
    with torch.enable_grad():
        log_score = f.logsigmoid(at) if case["scores"] == "sigmoid" else torch.log_softmax(at, 1)
    score = torch.sigmoid(l) if case["scores"] == "sigmoid" else log_score.detach().exp()
    c = score + (0.0 if s["bias"] is None else s["bias"].double())
    c = c.masked_fill(dead, -math.inf)
    ids = torch.arange(E, device=l.device).expand(T, E)
    if case["top_groups"] < G:
        of_group = []
        for g in c.split(E // G, dim=1):
            first = g.amax(1)
            if case["group_top"] == 2:
                second = g.scatter(1, g.argmax(1, keepdim=True), -math.inf).amax(1)
                first = first + second.masked_fill(second == -math.inf, 0.0)
            of_group.append(first)
        of_group = torch.stack(of_group, 1)
        # (a group stays if fewer than top_groups come before it)
        mine, other = of_group[:, :, None], of_group[:, None, :]
        number = torch.arange(G, device=l.device)
        before = ((other > mine) | ((other == mine) & (number[None, None, :] < number[None, :, None]))).sum(2)
        c = c.masked_fill((before >= case["top_groups"])[:, ids[0] // (E // G)], -math.inf)
    chosen = []
    for _ in range(k):
        best = c.amax(1, keepdim=True)
        first = torch.where(c == best, ids, E).amin(1)
        chosen.append(torch.where(best[:, 0] == -math.inf, -1, first))
        c = c.scatter(1, first[:, None], -math.inf)
    chosen = torch.stack(chosen, 1)
    live = chosen >= 0
    with torch.enable_grad():
        picked = torch.gather(log_score, 1, chosen.clamp(min=0))
        if case["normalise"]:
            picked = torch.log_softmax(picked.masked_fill(~live, -1e300), 1)
        w = torch.where(live, case["scale"] * picked.exp(), 0.0)
        out = [chosen.to(torch.int32), w.detach()]
        if case["train"]:
            d, = torch.autograd.grad((w * s["d_weights"].double()).sum(), at)
            out.append(d.masked_fill(~live.any(1, keepdim=True), 0.0))
    return out


def _exact_activation(z, name):
    f = torch.nn.functional
    if name == "swiglu":
        half = z.shape[-1] // 2
        return f.silu(z[..., :half]) * z[..., half:]
    return {"none": lambda v: v, "relu": f.relu, "gelu": f.gelu, "silu": f.silu}[name](z)


def _exact_int8(s):
    case, W, x = s["case"], s["W"], s["X"].double()
    T, k, E, N = case["tokens"], case["top_k"], case["experts"], case["d_out"]
    rows = T * k
    # (the scale is a float32 number by definition)
    scale = (x.abs().amax(1) / 127.0).float().double()
    q = x / scale.clamp(min=1e-300)[:, None]
    low = torch.floor(q)
    up = (q - low > 0.5) | ((q - low == 0.5) & (low % 2.0 != 0.0))
    q = torch.minimum(torch.maximum(low + up, torch.tensor(-127.0, device=q.device, dtype=q.dtype)), torch.tensor(127.0, device=q.device, dtype=q.dtype))
    Y = torch.zeros(rows, N, dtype=torch.float64, device=x.device)
    flat = s["experts"].reshape(-1) if E else torch.zeros(rows, dtype=torch.int32, device=x.device)
    to_of = s["order"][2].long() if E else torch.arange(rows, device=x.device)
    for e in range(max(E, 1)):
        mine = torch.nonzero(flat == e).flatten()
        if not mine.numel():
            continue
        to, token = to_of[mine], mine // k
        w = W[e].double() * s["W_scales"][e].double()[:, None]
        z = torch.matmul(w, (q[token] * scale[token][:, None]).t()).t()
        if s["bias"] is not None:
            z = z + s["bias"][e].double()
        y = _exact_activation(z, case["activation"])
        Y[to] = y if s["residual"] is None else y + s["residual"].double()[to]
    return [scale, Y]


def _exact_kept(X):
    """The same with the exponents from a table of the borders between them."""
    n, w = X.shape
    least = -24 if X.dtype is torch.float16 else -126
    powers = torch.arange(least, 128, device=X.device)
    borders = 127.5 * torch.exp2(powers.double())
    kept, bytes_ = [], []
    for part in X.double().split(_BLOCK, dim=1):
        which = torch.searchsorted(borders, part.abs().amax(1).contiguous(), right=True)
        unit = torch.exp2(powers[which].double())[:, None]
        q = part / unit
        low = torch.floor(q)
        q = low + ((q - low > 0.5) | ((q - low == 0.5) & (low % 2.0 != 0.0)))
        past = (q * unit).abs() > torch.finfo(X.dtype).max
        kept.append(torch.where(past, q - torch.sign(q), q) * unit)
        bytes_.append(powers[which] + 127)
    return torch.cat(kept, 1), torch.stack(bytes_, 1).to(torch.uint8)


def _exact_rows8(s):
    kept, exponents = _exact_kept(s["X"])
    return [exponents, _exact_activation(kept, s["case"]["activation"])]


def _exact_backward8(s):
    case = s["case"]
    k, E, D = case["top_k"], case["experts"], case["width"]
    (X, _), (pre, _) = _exact_kept(s["X"]), _exact_kept(s["pre"])
    flat, to_of = s["experts"].reshape(-1), s["order"][2].long()
    d_pre = torch.zeros_like(pre)
    dW = torch.zeros(E, pre.shape[1], D, dtype=torch.float64, device=X.device)
    db = torch.zeros(E, pre.shape[1], dtype=torch.float64, device=X.device)
    for e in range(E):
        mine = torch.nonzero(flat == e).flatten()
        if not mine.numel():
            continue
        to = to_of[mine]
        d = torch.matmul(s["W2"][e].double().t(), s["d_ys"].double()[to].t()).t()
        with torch.enable_grad():
            at = pre[to].requires_grad_()
            d_pre[to], = torch.autograd.grad(_exact_activation(at, case["activation"]), at, d)
        dz = s["d_z"].double()[to]
        dW[e] = torch.matmul(X[mine // k].t(), dz).t()
        db[e] = torch.ones(1, mine.numel(), dtype=torch.float64, device=X.device).matmul(dz)[0]
    return [d_pre, dW, db]


def exact(case, seed):
    s = prepare(case, seed)
    return {"route": _exact_route, "int8": _exact_int8, "rows8": _exact_rows8, "backward8": _exact_backward8}[case["op"]](s)
