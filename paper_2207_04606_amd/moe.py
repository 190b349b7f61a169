"""The operators of a mixture-of-experts layer: ctypes binding of the sptir_moe_* entry points (argument marshalling only).

Tensors are float32, float16 or bfloat16, all of a call the same; router weights, their gradient and sums are float32, ids
int32.  A matrix may have any row stride, its rows have to be contiguous.  Outputs are given by the caller and overwritten.
"""
from __future__ import annotations

import contextlib
import ctypes

import torch

from .binding import SPTIR_OK, SptirError, _dev, _stream_ptr, load_library

TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3, "swiglu": 4}
_NULL = (None, 0)
_NOTHING = contextlib.nullcontext()


class _Routing(ctypes.Structure):
    _fields_ = [("n_tokens", ctypes.c_int32), ("top_k", ctypes.c_int32), ("n_experts", ctypes.c_int32),
                ("expert_ptr", ctypes.c_void_p), ("entry_of", ctypes.c_void_p), ("slot_of", ctypes.c_void_p)]


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
        routing = ctypes.POINTER(_Routing)
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
        for name in ("route", "route_backward", "sort", "gather", "combine", "combine_backward", "product", "product_dx",
                     "product_dw"):
            getattr(lib, "sptir_moe_" + name).restype = ctypes.c_int
        lib.sptir_moe_sort_workspace.restype = lib.sptir_moe_product_dw_workspace.restype = i64
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


_PRODUCT_SIZE, _PRODUCT_DX_SIZE, _PRODUCT_DW_SIZE = (ctypes.sizeof(s) for s in (_Product, _ProductDx, _ProductDw))
EXPORTED_SYMBOLS = ("sptir_moe_route", "sptir_moe_route_backward", "sptir_moe_sort", "sptir_moe_sort_workspace", "sptir_moe_gather",
                    "sptir_moe_combine", "sptir_moe_combine_backward", "sptir_moe_product", "sptir_moe_product_dx",
                    "sptir_moe_product_dw", "sptir_moe_product_dw_workspace")
