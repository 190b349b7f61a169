"""The operators of a mixture-of-experts layer: ctypes binding of the sptir_moe_* entry points (argument marshalling only).

Tensors are float32, float16 or bfloat16, all of a call the same; router weights, their gradient and sums are float32, ids
int32.  A matrix may have any row stride, its rows have to be contiguous.  Outputs are given by the caller and overwritten.

Two forms of 8 bits: `sptir_moe_quantise` and `sptir_moe_product_int8` multiply whole numbers with a scale for each row of X and of W
(serving); `sptir_moe_pack`, `sptir_moe_unpack` and the `_packed` gradients keep activations between the forward and the backward
pass with a power of two for every BLOCK columns (training).
"""
from __future__ import annotations

import contextlib
import ctypes

import torch

from .binding import SPTIR_OK, SptirError, _dev, _stream_ptr, load_library

TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
SCORES = {"softmax": 0, "sigmoid": 1}
BLOCK = 32  # columns of a packed row that share an exponent
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3, "swiglu": 4}
_NULL = (None, 0)
_NOTHING = contextlib.nullcontext()


class _Routing(ctypes.Structure):
    _fields_ = [("n_tokens", ctypes.c_int32), ("top_k", ctypes.c_int32), ("n_experts", ctypes.c_int32),
                ("expert_ptr", ctypes.c_void_p), ("entry_of", ctypes.c_void_p), ("slot_of", ctypes.c_void_p)]


class _Scoring(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_int32), ("score", ctypes.c_int32), ("normalise", ctypes.c_int32),
                ("n_groups", ctypes.c_int32), ("top_groups", ctypes.c_int32), ("group_top", ctypes.c_int32),
                ("scale", ctypes.c_float), ("bias", ctypes.c_void_p)]


class _Product(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_int32), ("type", ctypes.c_int32), ("activation", ctypes.c_int32),
                ("gather", ctypes.c_int32), ("d_in", ctypes.c_int32), ("d_out", ctypes.c_int32), ("n_rows", ctypes.c_int64),
                ("X", ctypes.c_void_p), ("ldx", ctypes.c_int64),
                ("W", ctypes.c_void_p), ("ldw", ctypes.c_int64), ("w_stride", ctypes.c_int64),
                ("bias", ctypes.c_void_p), ("bias_stride", ctypes.c_int64),
                ("residual", ctypes.c_void_p), ("ld_residual", ctypes.c_int64),
                ("pre", ctypes.c_void_p), ("ld_pre", ctypes.c_int64), ("Y", ctypes.c_void_p), ("ldy", ctypes.c_int64)]


class _ProductDx(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_int32), ("type", ctypes.c_int32), ("activation", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("d_in", ctypes.c_int32), ("d_z", ctypes.c_int32), ("n_rows", ctypes.c_int64),
                ("dZ", ctypes.c_void_p), ("ld_dz", ctypes.c_int64),
                ("W", ctypes.c_void_p), ("ldw", ctypes.c_int64), ("w_stride", ctypes.c_int64),
                ("pre", ctypes.c_void_p), ("ld_pre", ctypes.c_int64), ("dX", ctypes.c_void_p), ("ld_dx", ctypes.c_int64)]


class _ProductDw(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_int32), ("type", ctypes.c_int32), ("gather", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("d_in", ctypes.c_int32), ("d_z", ctypes.c_int32), ("n_rows", ctypes.c_int64),
                ("dZ", ctypes.c_void_p), ("ld_dz", ctypes.c_int64), ("X", ctypes.c_void_p), ("ldx", ctypes.c_int64),
                ("dW", ctypes.c_void_p), ("ld_dw", ctypes.c_int64), ("dw_stride", ctypes.c_int64),
                ("db", ctypes.c_void_p), ("db_stride", ctypes.c_int64),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_int64)]


_ready = None


def _library():
    global _ready
    if _ready is None:
        lib = load_library()
        i32, i64, ptr = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p
        routing, scoring = ctypes.POINTER(_Routing), ctypes.POINTER(_Scoring)
        lib.sptir_moe_route.argtypes = [ptr, i32, i64, i32, i32, i32, i32, ptr, ptr, ptr]
        lib.sptir_moe_route_backward.argtypes = [ptr, i32, i64, i32, i32, i32, i32, ptr, ptr, ptr, ptr, i64, ptr]
        lib.sptir_moe_sort_workspace.argtypes = [i64, i32]
        lib.sptir_moe_sort.argtypes = [ptr, i32, i32, i32, ptr, ptr, ptr, ptr, i64, ptr]
        lib.sptir_moe_gather.argtypes = [routing, i32, i32, ptr, i64, ptr, ptr, i64, ptr]
        lib.sptir_moe_combine.argtypes = [routing, i32, i32, ptr, i64, ptr, ptr, i64, ptr, i64, ptr]
        lib.sptir_moe_combine_backward.argtypes = [routing, i32, i32, ptr, i64, ptr, i64, ptr, ptr, i64, ptr, ptr]
        lib.sptir_moe_product.argtypes = [routing, ctypes.POINTER(_Product), ptr]
        lib.sptir_moe_product_dx.argtypes = [routing, ctypes.POINTER(_ProductDx), ptr]
        lib.sptir_moe_product_dw_workspace.argtypes = [i64, i32, i32, i32]
        lib.sptir_moe_product_dw.argtypes = [routing, ctypes.POINTER(_ProductDw), ptr]
        lib.sptir_moe_route_groups.argtypes = [ptr, i32, i64, i32, i32, i32, scoring, ptr, ptr, ptr]
        lib.sptir_moe_route_groups_backward.argtypes = [ptr, i32, i64, i32, i32, i32, scoring, ptr, ptr, ptr, ptr, i64, ptr]
        lib.sptir_moe_quantise.argtypes = [i32, i32, i64, ptr, i64, ptr, i64, ptr, ptr]
        lib.sptir_moe_product_int8.argtypes = [routing, ctypes.POINTER(_Product), ptr, ptr, i64, ptr]
        lib.sptir_moe_pack.argtypes = [i32, i32, i64, ptr, i64, ptr, i64, ptr, i64, ptr]
        lib.sptir_moe_unpack.argtypes = [i32, i32, i32, i64, ptr, i64, ptr, i64, ptr, i64, ptr]
        lib.sptir_moe_product_dx_packed.argtypes = [routing, ctypes.POINTER(_ProductDx), ptr, i64, ptr]
        lib.sptir_moe_product_dw_packed_workspace.argtypes = [i32, i64, i64, i32, i32, i32]
        lib.sptir_moe_product_dw_packed.argtypes = [routing, ctypes.POINTER(_ProductDw), ptr, i64, ptr]
        for name in EXPORTED_SYMBOLS:
            getattr(lib, name).restype = i64 if name.endswith("_workspace") else ctypes.c_int
        _ready = lib
    return _ready


def _check(status, where):
    if status != SPTIR_OK:
        raise SptirError(status, where)


def _matrix(t, dtype, rows, cols, what):
    """(pointer, row stride) of a matrix with contiguous rows; (None, 0) for None."""
    if t is None:
        return _NULL
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what} must be a CUDA/HIP tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{what} must have dtype {dtype}, got {t.dtype}")
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != cols:
        raise ValueError(f"{what} must be [{rows}, {cols}], got {list(t.shape)}")
    ld, one = t.stride()
    if cols > 1 and one != 1:
        raise ValueError(f"the rows of {what} must be contiguous")
    if rows <= 1:
        ld = max(ld, cols)  # (torch gives such a matrix any stride)
    if ld < cols:
        raise ValueError(f"the rows of {what} must not overlap")
    return t.data_ptr() or None, ld


def _type(t, what):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what} must be a CUDA/HIP tensor")
    if t.dtype not in TYPES:
        raise TypeError(f"{what} must be float32, float16 or bfloat16, got {t.dtype}")
    return TYPES[t.dtype]


def _per_entry(t, dtype, shape, what):
    if t is None:
        return None
    _dev(t, dtype, what)
    if t.dim() != 2 or t.shape[0] != shape[0] or t.shape[1] != shape[1]:
        raise ValueError(f"{what} must be {list(shape)}, got {list(t.shape)}")
    return t.data_ptr() or None


def _under(stream):
    """The context in which memory for a call on `stream` is allocated.  The caching allocator orders a block's reuse against the
    stream it is taken under only: one taken under the current stream may still be in use there when the call's kernels begin."""
    if stream is None:
        return _NOTHING
    if not isinstance(stream, torch.cuda.Stream):
        number = int(getattr(stream, "cuda_stream", stream))
        stream = torch.cuda.ExternalStream(number) if number else torch.cuda.default_stream()
    return torch.cuda.stream(stream)


def _workspace(nbytes, stream):
    """Device memory for one call."""
    if nbytes == 0:
        return None
    with _under(stream):
        return torch.empty(nbytes, dtype=torch.uint8, device="cuda")


class MoeRouting:
    """The entries in the order of the experts: expert_ptr [E + 1], entry_of [T * k] and slot_of [T * k], int32 tensors."""

    def __init__(self, n_tokens, top_k, n_experts, expert_ptr, entry_of, slot_of):
        self.n_tokens, self.top_k, self.n_experts = n_tokens, top_k, n_experts
        self.expert_ptr, self.entry_of, self.slot_of = expert_ptr, entry_of, slot_of
        for t, n, what in ((expert_ptr, n_experts + 1, "expert_ptr"), (entry_of, n_tokens * top_k, "entry_of"),
                           (slot_of, n_tokens * top_k, "slot_of")):
            _dev(t, torch.int32, what)
            if t.numel() != n:
                raise ValueError(f"{what} must have {n} elements")
        self._struct = _Routing(n_tokens, top_k, n_experts, expert_ptr.data_ptr(), entry_of.data_ptr() or None,
                                slot_of.data_ptr() or None)
        self._ref = ctypes.byref(self._struct)

    @property
    def n_rows(self):
        return self.n_tokens * self.top_k


def sptir_moe_route(logits, experts, weights, normalise: bool = True, stream=None) -> None:
    """experts [T, k] and weights [T, k] from logits [T, E]: the k largest of a token and their softmax."""
    lib = _ready or _library()
    kind = _type(logits, "logits")
    if logits.dim() != 2 or experts.dim() != 2:
        raise ValueError("logits and experts must be 2-D")
    T, E = logits.shape
    k = experts.shape[1]
    l, ld = _matrix(logits, logits.dtype, T, E, "logits")
    st = lib.sptir_moe_route(l, kind, ld, T, E, k, int(normalise), _per_entry(experts, torch.int32, (T, k), "experts"),
                             _per_entry(weights, torch.float32, (T, k), "weights"), _stream_ptr(stream))
    _check(st, "sptir_moe_route")


def sptir_moe_route_backward(logits, experts, weights, d_weights, d_logits, normalise: bool = True, stream=None) -> None:
    """d_logits [T, E] from d_weights [T, k]; experts and weights as sptir_moe_route gave them."""
    lib = _ready or _library()
    kind = _type(logits, "logits")
    if logits.dim() != 2 or experts.dim() != 2:
        raise ValueError("logits and experts must be 2-D")
    T, E = logits.shape
    k = experts.shape[1]
    l, ld = _matrix(logits, logits.dtype, T, E, "logits")
    d, ldd = _matrix(d_logits, logits.dtype, T, E, "d_logits")
    st = lib.sptir_moe_route_backward(l, kind, ld, T, E, k, int(normalise), _per_entry(experts, torch.int32, (T, k), "experts"),
                                      _per_entry(weights, torch.float32, (T, k), "weights"),
                                      _per_entry(d_weights, torch.float32, (T, k), "d_weights"), d, ldd, _stream_ptr(stream))
    _check(st, "sptir_moe_route_backward")


def sptir_moe_route_groups(logits, experts, weights, scores: str = "softmax", bias=None, n_groups: int = 1, top_groups: int = 1,
                           group_top: int = 1, normalise: bool = True, scale: float = 1.0, stream=None) -> None:
    """experts [T, k] and weights [T, k] from logits [T, E]: the k largest scores ("softmax" or "sigmoid") plus bias [E], float32,
    out of the top_groups best of n_groups groups of neighbouring experts, a group's score being the sum of its group_top (1 or 2) largest.
    The weights are the scores without the bias, normalised to a sum of 1 if asked for, times scale."""
    lib = _ready or _library()
    kind = _type(logits, "logits")
    if logits.dim() != 2 or experts.dim() != 2:
        raise ValueError("logits and experts must be 2-D")
    T, E = logits.shape
    k = experts.shape[1]
    l, ld = _matrix(logits, logits.dtype, T, E, "logits")
    if bias is not None:
        _dev(bias, torch.float32, "bias")
        if bias.dim() != 1 or bias.shape[0] != E:
            raise ValueError(f"bias must be [{E}], got {list(bias.shape)}")
    how = _Scoring(_SCORING_SIZE, _score(scores), int(normalise), n_groups, top_groups, group_top, scale,
                   bias.data_ptr() if bias is not None else None)
    _here(logits, experts, weights, bias)
    st = lib.sptir_moe_route_groups(l, kind, ld, T, E, k, ctypes.byref(how), _per_entry(experts, torch.int32, (T, k), "experts"),
                                    _per_entry(weights, torch.float32, (T, k), "weights"), _stream_ptr(stream))
    _check(st, "sptir_moe_route_groups")


def sptir_moe_route_groups_backward(logits, experts, weights, d_weights, d_logits, scores: str = "softmax", normalise: bool = True,
                                    scale: float = 1.0, stream=None) -> None:
    """d_logits [T, E] from d_weights [T, k]; experts, weights and what they were made with as in sptir_moe_route_groups (bias and
    groups have no part in the gradient)."""
    lib = _ready or _library()
    kind = _type(logits, "logits")
    if logits.dim() != 2 or experts.dim() != 2:
        raise ValueError("logits and experts must be 2-D")
    T, E = logits.shape
    k = experts.shape[1]
    l, ld = _matrix(logits, logits.dtype, T, E, "logits")
    d, ldd = _matrix(d_logits, logits.dtype, T, E, "d_logits")
    how = _Scoring(_SCORING_SIZE, _score(scores), int(normalise), 1, 1, 1, scale, None)
    _here(logits, experts, weights, d_weights, d_logits)
    st = lib.sptir_moe_route_groups_backward(l, kind, ld, T, E, k, ctypes.byref(how),
                                             _per_entry(experts, torch.int32, (T, k), "experts"),
                                             _per_entry(weights, torch.float32, (T, k), "weights"),
                                             _per_entry(d_weights, torch.float32, (T, k), "d_weights"), d, ldd, _stream_ptr(stream))
    _check(st, "sptir_moe_route_groups_backward")


def sptir_moe_sort(experts, n_experts: int, routing: MoeRouting | None = None, stream=None) -> MoeRouting:
    """Sorts the entries of experts [T, k] by expert; entries outside 0 .. n_experts - 1 are dropped.  `routing`: an earlier
    result for the same sizes, whose arrays are overwritten."""
    lib = _ready or _library()
    _dev(experts, torch.int32, "experts")
    if experts.dim() != 2:
        raise ValueError("experts must be 2-D")
    T, k = experts.shape
    n = T * k
    if routing is None:
        with _under(stream):
            new = [torch.empty(m, dtype=torch.int32, device=experts.device) for m in (max(int(n_experts), 0) + 1, n, n)]
        if stream is not None:  # (the caller will use them under the current stream)
            for t in new:
                t.record_stream(torch.cuda.current_stream())
        routing = MoeRouting(T, k, int(n_experts), *new)
    elif (routing.n_tokens, routing.top_k, routing.n_experts) != (T, k, n_experts):
        raise ValueError("routing has arrays of other sizes")
    s = routing._struct
    ws = _workspace(lib.sptir_moe_sort_workspace(n, n_experts), stream)
    st = lib.sptir_moe_sort(experts.data_ptr() or None, T, k, n_experts, s.expert_ptr, s.entry_of, s.slot_of,
                            ws.data_ptr() if ws is not None else None, ws.numel() if ws is not None else 0, _stream_ptr(stream))
    _check(st, "sptir_moe_sort")
    return routing


def sptir_moe_gather(routing: MoeRouting, X, Xs, weights=None, stream=None) -> None:
    """Xs [T * k, width], in sorted order, from X [T, width]; with weights [T, k] times the entry's weight."""
    lib = _ready or _library()
    kind = _type(X, "X")
    width = X.shape[-1]
    x, ldx = _matrix(X, X.dtype, routing.n_tokens, width, "X")
    o, ldo = _matrix(Xs, X.dtype, routing.n_rows, width, "Xs")
    w = _per_entry(weights, torch.float32, (routing.n_tokens, routing.top_k), "weights")
    _check(lib.sptir_moe_gather(routing._ref, kind, width, x, ldx, w, o, ldo, _stream_ptr(stream)), "sptir_moe_gather")


def sptir_moe_combine(routing: MoeRouting, Ys, Y, weights=None, residual=None, stream=None) -> None:
    """Y [T, width] = residual + the sum over a token's entries of weight times its row of Ys [T * k, width]."""
    lib = _ready or _library()
    kind = _type(Ys, "Ys")
    width = Ys.shape[-1]
    ys, ldys = _matrix(Ys, Ys.dtype, routing.n_rows, width, "Ys")
    r, ldr = _matrix(residual, Ys.dtype, routing.n_tokens, width, "residual")
    y, ldy = _matrix(Y, Ys.dtype, routing.n_tokens, width, "Y")
    w = _per_entry(weights, torch.float32, (routing.n_tokens, routing.top_k), "weights")
    _check(lib.sptir_moe_combine(routing._ref, kind, width, ys, ldys, w, r, ldr, y, ldy, _stream_ptr(stream)),
           "sptir_moe_combine")


def sptir_moe_combine_backward(routing: MoeRouting, dY, Ys, weights, dYs, d_weights=None, stream=None) -> None:
    """The gradients of sptir_moe_combine: dYs [T * k, width] and, if wanted, d_weights [T, k] (Ys is read for these only)."""
    lib = _ready or _library()
    kind = _type(dY, "dY")
    width = dY.shape[-1]
    shape = (routing.n_tokens, routing.top_k)
    d, ldd = _matrix(dY, dY.dtype, routing.n_tokens, width, "dY")
    ys, ldys = _matrix(Ys, dY.dtype, routing.n_rows, width, "Ys")
    if d_weights is not None and Ys is None:
        raise ValueError("d_weights needs Ys")
    o, ldo = _matrix(dYs, dY.dtype, routing.n_rows, width, "dYs")
    st = lib.sptir_moe_combine_backward(routing._ref, kind, width, d, ldd, ys, ldys,
                                        _per_entry(weights, torch.float32, shape, "weights"), o, ldo,
                                        _per_entry(d_weights, torch.float32, shape, "d_weights"), _stream_ptr(stream))
    _check(st, "sptir_moe_combine_backward")


def _here(*tensors, routing=None):
    """A call runs on the current device, and so are its tensors and the arrays of its routing."""
    device = torch.cuda.current_device()
    for t in tensors if routing is None else (*tensors, routing.expert_ptr, routing.entry_of):
        if t is not None and t.get_device() != device:
            raise ValueError(f"a tensor is on {t.device}, the current device is {device}")


def _vector(t, n, what):
    _dev(t, torch.float32, what)
    if t.dim() != 1 or t.shape[0] != n:
        raise ValueError(f"{what} must be [{n}], got {list(t.shape)}")
    return t.data_ptr() or None


def _experts_matrix(W, dtype, n_experts, what):
    """(pointer, row stride, stride of an expert, rows, columns) of [E, rows, columns], or of [rows, columns] for one."""
    if not isinstance(W, torch.Tensor) or not W.is_cuda:
        raise TypeError(f"{what} must be a CUDA/HIP tensor")
    if W.dtype is not dtype:
        raise TypeError(f"{what} must have dtype {dtype}, got {W.dtype}")
    shape, stride = W.shape, W.stride()
    if len(shape) == 2 and n_experts == 1:
        shape, stride = (1, *shape), (0, *stride)
    if len(shape) != 3 or shape[0] != n_experts:
        raise ValueError(f"{what} must be [{n_experts}, rows, columns], got {list(W.shape)}")
    if shape[2] > 1 and stride[2] != 1:
        raise ValueError(f"the rows of {what} must be contiguous")
    ld = max(stride[1], shape[2]) if shape[1] <= 1 else stride[1]
    return W.data_ptr() or None, ld, stride[0], shape[1], shape[2]


def _experts_vector(b, dtype, n_experts, n, what):
    if b is None:
        return _NULL
    if not isinstance(b, torch.Tensor) or not b.is_cuda:
        raise TypeError(f"{what} must be a CUDA/HIP tensor")
    if b.dtype is not dtype:
        raise TypeError(f"{what} must have dtype {dtype}, got {b.dtype}")
    shape, stride = b.shape, b.stride()
    if len(shape) == 1 and n_experts == 1:
        shape, stride = (1, *shape), (0, *stride)
    if len(shape) != 2 or shape[0] != n_experts or shape[1] != n or (n > 1 and stride[1] != 1):
        raise ValueError(f"{what} must be [{n_experts}, {n}] with contiguous rows")
    return b.data_ptr() or None, stride[0]


def _score(name):
    if name not in SCORES:
        raise ValueError(f"unknown scores {name!r}; one of {sorted(SCORES)}")
    return SCORES[name]


def _activation(name):
    if name not in ACTIVATIONS:
        raise ValueError(f"unknown activation {name!r}; one of {sorted(ACTIVATIONS)}")
    return ACTIVATIONS[name]


def sptir_moe_product(routing: MoeRouting | None, X, W, Y, bias=None, residual=None, pre=None, activation: str = "none",
                      gather: bool = False, stream=None) -> None:
    """Y[s] = act(W[e] x + bias[e]) + residual[s] for every row s of every expert e; W [E, wide, d_in].

    x is X[s], or with `gather` the row of the entry's token (X [T, d_in]).  pre [rows, wide] receives W[e] x + bias[e].
    routing None: one expert with all rows (W may be 2-D and bias 1-D)."""
    lib = _ready or _library()
    kind, act = _type(X, "X"), _activation(activation)
    dtype = X.dtype
    E = routing.n_experts if routing is not None else 1
    w, ldw, w_stride, wide, d_in = _experts_matrix(W, dtype, E, "W")
    if act == 4 and wide % 2:
        raise ValueError("the W of swiglu has an even number of rows")
    d_out = wide // 2 if act == 4 else wide
    if gather and routing is None:
        raise ValueError("gather needs a routing")
    rows = routing.n_rows if routing is not None else X.shape[0]
    x, ldx = _matrix(X, dtype, routing.n_tokens if gather else rows, d_in, "X")
    b, b_stride = _experts_vector(bias, dtype, E, wide, "bias")
    r, ldr = _matrix(residual, dtype, rows, d_out, "residual")
    z, ldz = _matrix(pre, dtype, rows, wide, "pre")
    y, ldy = _matrix(Y, dtype, rows, d_out, "Y")
    q = _Product(_PRODUCT_SIZE, kind, act, 1 if gather else 0, d_in, d_out, rows, x, ldx, w, ldw, w_stride, b, b_stride, r, ldr,
                 z, ldz, y, ldy)
    _check(lib.sptir_moe_product(routing._ref if routing is not None else None, ctypes.byref(q), _stream_ptr(stream)),
           "sptir_moe_product")


def sptir_moe_product_dx(routing: MoeRouting | None, dZ, W, dX, pre=None, activation: str = "none", stream=None) -> None:
    """dX[s] = W[e]^T dZ[s]; with an activation times its derivative at pre[s], the z of the product that made x."""
    lib = _ready or _library()
    kind, act = _type(dZ, "dZ"), _activation(activation)
    dtype = dZ.dtype
    E = routing.n_experts if routing is not None else 1
    w, ldw, w_stride, d_z, d_in = _experts_matrix(W, dtype, E, "W")
    rows = routing.n_rows if routing is not None else dZ.shape[0]
    wide = 2 * d_in if act == 4 else d_in
    if act and pre is None:
        raise ValueError("an activation needs pre")
    dz, ld_dz = _matrix(dZ, dtype, rows, d_z, "dZ")
    z, ldz = _matrix(pre if act else None, dtype, rows, wide, "pre")
    dx, ld_dx = _matrix(dX, dtype, rows, wide, "dX")
    q = _ProductDx(_PRODUCT_DX_SIZE, kind, act, 0, d_in, d_z, rows, dz, ld_dz, w, ldw, w_stride, z, ldz, dx, ld_dx)
    _check(lib.sptir_moe_product_dx(routing._ref if routing is not None else None, ctypes.byref(q), _stream_ptr(stream)),
           "sptir_moe_product_dx")


def sptir_moe_product_dw(routing: MoeRouting | None, dZ, X, dW, db=None, gather: bool = False, stream=None) -> None:
    """dW[e] = the sum over expert e's rows of dZ[s] x^T, and db[e] that of dZ[s]; dW [E, d_z, d_in]."""
    lib = _ready or _library()
    kind = _type(dZ, "dZ")
    dtype = dZ.dtype
    E = routing.n_experts if routing is not None else 1
    w, ldw, w_stride, d_z, d_in = _experts_matrix(dW, dtype, E, "dW")
    if gather and routing is None:
        raise ValueError("gather needs a routing")
    rows = routing.n_rows if routing is not None else dZ.shape[0]
    dz, ld_dz = _matrix(dZ, dtype, rows, d_z, "dZ")
    x, ldx = _matrix(X, dtype, routing.n_tokens if gather else rows, d_in, "X")
    b, b_stride = _experts_vector(db, dtype, E, d_z, "db")
    ws = _workspace(lib.sptir_moe_product_dw_workspace(rows, E, d_in, d_z), stream)
    q = _ProductDw(_PRODUCT_DW_SIZE, kind, 1 if gather else 0, 0, d_in, d_z, rows, dz, ld_dz, x, ldx, w, ldw, w_stride, b, b_stride,
                   ws.data_ptr() if ws is not None else None, ws.numel() if ws is not None else 0)
    _check(lib.sptir_moe_product_dw(routing._ref if routing is not None else None, ctypes.byref(q), _stream_ptr(stream)),
           "sptir_moe_product_dw")


def sptir_moe_quantise(X, Q, scales, stream=None) -> None:
    """Q (int8) and scales (float32) of the rows of X, float32, float16 or bfloat16: X[r] ~ Q[r] * scales[r], scales[r] = max |X[r]| / 127.
    X [rows, width] and scales [rows], or the weights of experts, X [E, rows, width] and scales [E, rows], whose matrices follow one another."""
    lib = _ready or _library()
    kind = _type(X, "X")
    if X.dim() == 3 and isinstance(Q, torch.Tensor) and Q.dim() == 3 and isinstance(scales, torch.Tensor) and scales.dim() == 2:
        if Q.shape != X.shape or scales.shape != X.shape[:2]:
            raise ValueError(f"Q must be {list(X.shape)} and scales {list(X.shape[:2])}")
        for t in (X, Q, scales):
            if not t.is_contiguous():
                raise ValueError("the matrices of experts and their scales must be contiguous")
        rows = X.shape[0] * X.shape[1]
        X, Q, scales = X.view(rows, X.shape[2]), Q.view(rows, X.shape[2]), scales.view(rows)
    if X.dim() != 2:
        raise ValueError("X must be [rows, width], or [E, rows, width] beside Q of the same shape")
    rows, width = X.shape
    x, ldx = _matrix(X, X.dtype, rows, width, "X")
    q, ldq = _matrix(Q, torch.int8, rows, width, "Q")
    s = _vector(scales, rows, "scales")
    _here(X, Q, scales)
    _check(lib.sptir_moe_quantise(kind, width, rows, x, ldx, q, ldq, s, _stream_ptr(stream)), "sptir_moe_quantise")


def sptir_moe_product_int8(routing: MoeRouting | None, X, x_scales, W, w_scales, Y, bias=None, residual=None, pre=None,
                           activation: str = "none", gather: bool = False, stream=None) -> None:
    """sptir_moe_product with int8 X and W: x stands for X's row times x_scales[row], W[e] for its rows times w_scales[e].
    Y, bias, residual and pre have one type, float32, float16 or bfloat16; the scales are float32, w_scales [E, wide]."""
    lib = _ready or _library()
    kind, act = _type(Y, "Y"), _activation(activation)
    dtype = Y.dtype
    E = routing.n_experts if routing is not None else 1
    w, ldw, w_stride, wide, d_in = _experts_matrix(W, torch.int8, E, "W")
    if act == 4 and wide % 2:
        raise ValueError("the W of swiglu has an even number of rows")
    d_out = wide // 2 if act == 4 else wide
    if gather and routing is None:
        raise ValueError("gather needs a routing")
    rows = routing.n_rows if routing is not None else Y.shape[0]
    x_rows = routing.n_tokens if gather else rows
    x, ldx = _matrix(X, torch.int8, x_rows, d_in, "X")
    ws, ws_stride = _experts_vector(w_scales, torch.float32, E, wide, "w_scales")
    b, b_stride = _experts_vector(bias, dtype, E, wide, "bias")
    r, ldr = _matrix(residual, dtype, rows, d_out, "residual")
    z, ldz = _matrix(pre, dtype, rows, wide, "pre")
    y, ldy = _matrix(Y, dtype, rows, d_out, "Y")
    _here(X, x_scales, W, w_scales, Y, bias, residual, pre, routing=routing)
    q = _Product(_PRODUCT_SIZE, kind, act, 1 if gather else 0, d_in, d_out, rows, x, ldx, w, ldw, w_stride, b, b_stride, r, ldr,
                 z, ldz, y, ldy)
    st = lib.sptir_moe_product_int8(routing._ref if routing is not None else None, ctypes.byref(q), _vector(x_scales, x_rows, "x_scales"),
                                    ws, ws_stride, _stream_ptr(stream))
    _check(st, "sptir_moe_product_int8")


def _exponents(t, rows, width, what):
    return _matrix(t, torch.uint8, rows, -(-width // BLOCK), what)


def sptir_moe_pack(X, Q, exponents, stream=None) -> None:
    """Q (int8, as X) and exponents (uint8, [rows, ceil(width / BLOCK)]) of X [rows, width]: Q * 2^(exponents - 127)."""
    lib = _ready or _library()
    kind = _type(X, "X")
    if X.dim() != 2:
        raise ValueError("X must be 2-D")
    rows, width = X.shape
    x, ldx = _matrix(X, X.dtype, rows, width, "X")
    q, ldq = _matrix(Q, torch.int8, rows, width, "Q")
    e, lde = _exponents(exponents, rows, width, "exponents")
    _here(X, Q, exponents)
    _check(lib.sptir_moe_pack(kind, width, rows, x, ldx, q, ldq, e, lde, _stream_ptr(stream)), "sptir_moe_pack")


def sptir_moe_unpack(Q, exponents, Y, activation: str = "none", stream=None) -> None:
    """Y = act(what sptir_moe_pack kept of rows of Y's type), [rows, width], or [rows, width / 2] for swiglu."""
    lib = _ready or _library()
    kind, act = _type(Y, "Y"), _activation(activation)
    if Q.dim() != 2:
        raise ValueError("Q must be 2-D")
    rows, width = Q.shape
    if act == 4 and width % 2:
        raise ValueError("swiglu needs rows of an even width")
    q, ldq = _matrix(Q, torch.int8, rows, width, "Q")
    e, lde = _exponents(exponents, rows, width, "exponents")
    y, ldy = _matrix(Y, Y.dtype, rows, width // 2 if act == 4 else width, "Y")
    _here(Q, exponents, Y)
    _check(lib.sptir_moe_unpack(kind, act, width, rows, q, ldq, e, lde, y, ldy, _stream_ptr(stream)), "sptir_moe_unpack")


def sptir_moe_product_dx_packed(routing: MoeRouting | None, dZ, W, dX, pre, exponents, activation: str, stream=None) -> None:
    """sptir_moe_product_dx with the pre that sptir_moe_pack kept: int8 codes and their exponents."""
    lib = _ready or _library()
    kind, act = _type(dZ, "dZ"), _activation(activation)
    if not act:
        raise ValueError("without an activation there is no pre: sptir_moe_product_dx")
    dtype = dZ.dtype
    E = routing.n_experts if routing is not None else 1
    w, ldw, w_stride, d_z, d_in = _experts_matrix(W, dtype, E, "W")
    rows = routing.n_rows if routing is not None else dZ.shape[0]
    wide = 2 * d_in if act == 4 else d_in
    dz, ld_dz = _matrix(dZ, dtype, rows, d_z, "dZ")
    z, ldz = _matrix(pre, torch.int8, rows, wide, "pre")
    e, lde = _exponents(exponents, rows, wide, "exponents")
    dx, ld_dx = _matrix(dX, dtype, rows, wide, "dX")
    _here(dZ, W, dX, pre, exponents, routing=routing)
    q = _ProductDx(_PRODUCT_DX_SIZE, kind, act, 0, d_in, d_z, rows, dz, ld_dz, w, ldw, w_stride, z, ldz, dx, ld_dx)
    _check(lib.sptir_moe_product_dx_packed(routing._ref if routing is not None else None, ctypes.byref(q), e, lde, _stream_ptr(stream)),
           "sptir_moe_product_dx_packed")


def sptir_moe_product_dw_packed(routing: MoeRouting | None, dZ, X, exponents, dW, db=None, gather: bool = False, stream=None) -> None:
    """sptir_moe_product_dw with the X that sptir_moe_pack kept: int8 codes and their exponents.  (For the time of the call it takes
    memory for X in its type.)"""
    lib = _ready or _library()
    kind = _type(dZ, "dZ")
    dtype = dZ.dtype
    E = routing.n_experts if routing is not None else 1
    w, ldw, w_stride, d_z, d_in = _experts_matrix(dW, dtype, E, "dW")
    if gather and routing is None:
        raise ValueError("gather needs a routing")
    rows = routing.n_rows if routing is not None else dZ.shape[0]
    x_rows = routing.n_tokens if gather else rows
    dz, ld_dz = _matrix(dZ, dtype, rows, d_z, "dZ")
    x, ldx = _matrix(X, torch.int8, x_rows, d_in, "X")
    e, lde = _exponents(exponents, x_rows, d_in, "exponents")
    b, b_stride = _experts_vector(db, dtype, E, d_z, "db")
    _here(dZ, X, exponents, dW, db, routing=routing)
    ws = _workspace(lib.sptir_moe_product_dw_packed_workspace(kind, x_rows, rows, E, d_in, d_z), stream)
    q = _ProductDw(_PRODUCT_DW_SIZE, kind, 1 if gather else 0, 0, d_in, d_z, rows, dz, ld_dz, x, ldx, w, ldw, w_stride, b, b_stride,
                   ws.data_ptr() if ws is not None else None, ws.numel() if ws is not None else 0)
    _check(lib.sptir_moe_product_dw_packed(routing._ref if routing is not None else None, ctypes.byref(q), e, lde, _stream_ptr(stream)),
           "sptir_moe_product_dw_packed")


_PRODUCT_SIZE, _PRODUCT_DX_SIZE, _PRODUCT_DW_SIZE, _SCORING_SIZE = (ctypes.sizeof(s) for s in (_Product, _ProductDx, _ProductDw, _Scoring))
EXPORTED_SYMBOLS = ("sptir_moe_route", "sptir_moe_route_backward", "sptir_moe_route_groups", "sptir_moe_route_groups_backward",
                    "sptir_moe_sort", "sptir_moe_sort_workspace", "sptir_moe_gather", "sptir_moe_combine", "sptir_moe_combine_backward",
                    "sptir_moe_product", "sptir_moe_product_dx", "sptir_moe_product_dw", "sptir_moe_product_dw_workspace",
                    "sptir_moe_quantise", "sptir_moe_product_int8", "sptir_moe_pack", "sptir_moe_unpack", "sptir_moe_product_dx_packed",
                    "sptir_moe_product_dw_packed", "sptir_moe_product_dw_packed_workspace")
