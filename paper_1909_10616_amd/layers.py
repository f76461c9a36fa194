"""Layer operators of libgemmtune (include/gemmtune_layers.h), same names as the
C ABI: perceptron layers with their epilogue, their gradients, the routing of
tokens to experts and layers of experts.

Argument checks and marshalling only; every step runs in the library, on the
current stream (or ``stream``). Outputs and scratch memory come from PyTorch's
allocator, for that stream, unless given. Matrices may have any row stride;
their rows must be contiguous. Tensors given to a call on a stream other than
their own are the caller's to keep alive, as with any asynchronous call.

Outside autograd: results carry no graph, also where an operand requires a
gradient. The gradients are the _backward calls.
"""
from __future__ import annotations

import ctypes
import typing

from . import gemmtune as gt
from .gemmtune import BF16, F32, _check, _stream

ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
GATED = 16
SCORES = {"softmax": 0, "sigmoid": 1}

_i64, _i32, _P, _f32 = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_float


def _fields(text):
    kinds = {"i": _i32, "l": _i64, "p": _P, "f": _f32}
    return [(n, kinds[k]) for k, names in (part.split(":") for part in text.split(";"))
            for n in names.split()]


class gt_linear_args(ctypes.Structure):
    _fields_ = _fields("l:M N K;i:dtype act out_dtype reserved;p:X;l:ldx;p:W;l:ldw;p:bias R;l:ldr;"
                       "p:Y;l:ldy;p:P;l:ldp")


class gt_linear_grad_args(ctypes.Structure):
    _fields_ = _fields("l:M N K;i:dtype act dw_dtype reserved;p:dY;l:lddy;p:X;l:ldx;p:W;l:ldw;"
                       "p:P;l:ldp;p:dX;l:lddx;p:dW;l:lddw;p:db")


class gt_route_args(ctypes.Structure):
    _fields_ = _fields("l:T;i:E k groups keep dtype score renormalise;f:scale;p:logits;l:ldl;"
                       "p:bias weights experts offsets order place")


class gt_route_grad_args(ctypes.Structure):
    _fields_ = _fields("l:T;i:E k dtype score renormalise;f:scale;p:logits;l:ldl;"
                       "p:experts dweights dlogits;l:lddl")


class gt_experts_args(ctypes.Structure):
    _fields_ = _fields("l:T D H;i:E k dtype act;p:X;l:ldx;p:W1;l:ldw1 sw1;p:W2;l:ldw2 sw2;p:b1 b2 R;"
                       "l:ldr;p:Y;l:ldy;p:P;l:ldp;p:weights offsets order place")


class gt_experts_grad_args(ctypes.Structure):
    _fields_ = _fields("l:T D H;i:E k dtype act;p:dY;l:lddy;p:X;l:ldx;p:W1;l:ldw1 sw1;p:W2;"
                       "l:ldw2 sw2;p:b2 P;l:ldp;p:weights offsets order place dX;l:lddx;"
                       "p:dW1 dW2 db1 db2 dweights")


# entry point → its argument structure; those with a scratch have a _workspace
EXPORTS = {"gt_linear": gt_linear_args, "gt_linear_backward": gt_linear_grad_args,
           "gt_route": gt_route_args, "gt_route_backward": gt_route_grad_args,
           "gt_experts": gt_experts_args, "gt_experts_backward": gt_experts_grad_args}
NO_SCRATCH = ("gt_route_backward",)


class Route(typing.NamedTuple):
    """What gt_route gives: the experts of every token and their weights, and the
    lists of the experts' rows (entry t·k + s is slot s of token t)."""
    weights: typing.Any   # float32 [T, k]
    experts: typing.Any   # int32 [T, k], −1: none
    offsets: typing.Any   # int32 [E + 1]
    order: typing.Any     # int32 [T·k], entries sorted by expert, then −1
    place: typing.Any     # int32 [T, k], each entry's position in order, or −1


class ExpertGrads(typing.NamedTuple):
    dX: typing.Any
    dW1: typing.Any
    dW2: typing.Any
    db1: typing.Any
    db2: typing.Any
    dweights: typing.Any


_lib = None
_calls = {}   # entry point → its function and its scratch query


def lib():
    """The library with these entry points' signatures set."""
    global _lib
    if _lib is None:
        L = gt.lib()
        for name, args in EXPORTS.items():
            f = getattr(L, name)
            f.restype = ctypes.c_int
            if name in NO_SCRATCH:
                f.argtypes = [ctypes.POINTER(args), _P]
                continue
            f.argtypes = [ctypes.POINTER(args), _P, _i64, _P]
            w = getattr(L, name + "_workspace")
            w.argtypes, w.restype = [ctypes.POINTER(args), ctypes.POINTER(_i64)], ctypes.c_int
            _calls[name] = f, w
        _lib = L
    return _lib


def _act(act, gated):
    if act not in ACTS:
        raise ValueError(f"unknown activation {act!r}: one of {', '.join(ACTS)}")
    return ACTS[act] | (GATED if gated else 0)


def _type(t, name):
    import torch
    if t.dtype is torch.bfloat16:
        return BF16
    if t.dtype is torch.float32:
        return F32
    raise ValueError(f"{name} must be float32 or bfloat16")


def _tensor(t, name, like, shape, dtype=None):
    """A tensor of this shape, type (like's unless given) and like's device whose rows are
    contiguous; its pointer and row stride."""
    if t.dtype is not (dtype or like.dtype):
        raise ValueError(f"{name} must be {dtype or like.dtype}")
    if t.device != like.device:
        raise ValueError(f"{name} must be a GPU tensor on {like.device}")
    have = t.shape
    if have != shape:
        raise ValueError(f"{name} has shape {tuple(have)}, not {tuple(shape)}")
    st = t.stride()
    n = len(st)
    if n == 0 or (st[-1] != 1 and have[-1] != 1):
        raise ValueError(f"the rows of {name} must be contiguous")
    cols = have[-1]
    if n == 1:
        return t.data_ptr(), cols
    ld = st[-2]
    if ld < cols or cols == 0:
        if have[-2] != 1 and cols != 0:
            raise ValueError(f"the rows of {name} must not overlap")
        ld = max(ld, cols)
    return t.data_ptr(), ld


def _whole(t, name, like, shape, dtype=None):
    """As _tensor, contiguous as a whole; its pointer."""
    p, _ = _tensor(t, name, like, shape, dtype)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return p


def _pair(t, name, like, shape, dtype=None):
    return (None, 0) if t is None else _tensor(t, name, like, shape, dtype)


def _one(t, name, like, shape, dtype=None):
    return None if t is None else _whole(t, name, like, shape, dtype)


def _result_type(t, name, like):
    """The type of an output that is in like's type or in float32."""
    if t.dtype is not like.dtype and _type(t, name) != F32:
        raise ValueError(f"{name} must be {like.dtype} or torch.float32")
    return _type(t, name)


def _gpu(t, name, dims):
    if not t.is_cuda or t.dim() != dims:
        raise ValueError(f"{name} must be a GPU tensor of {dims} dimensions")


def _call(name, a, like, workspace, stream):
    """Runs an entry point on like's device, with scratch of its own unless given."""
    import torch
    L = lib()
    ref = ctypes.byref(a)
    with torch.cuda.device(like.device) if like.device.index != torch._C._cuda_getDevice() \
            else _NOTHING:
        if name in NO_SCRATCH:
            _check(getattr(L, name)(ref, _stream(stream)), name)
            return
        run, query = _calls[name]
        need = _i64()
        _check(query(ref, ctypes.byref(need)), name)
        n = need.value
        if n == 0:
            _check(run(ref, None, 0, _stream(stream)), name)
            return
        if workspace is None:
            workspace = _empty((n,), torch.uint8, like.device, stream)
        elif workspace.device != like.device or not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous, on the operands' device")
        _check(run(ref, workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                   _stream(stream)), name)


class _Nothing:
    def __enter__(self):
        return self

    def __exit__(self, *exc):
        return False


_NOTHING = _Nothing()


def _empty(shape, dtype, device, stream):
    """Memory for the stream the call runs on (PyTorch's allocator gives memory that is
    free in the order of one stream)."""
    import torch
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(int(stream), device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def workspace_bytes(name, args) -> int:
    """The scratch an entry point needs with these arguments (a structure of EXPORTS)."""
    need = _i64()
    _check(getattr(lib(), name + "_workspace")(ctypes.byref(args), ctypes.byref(need)), name)
    return need.value


def gt_linear(X, W, bias=None, residual=None, act="none", gated=False, Y=None, P=None,
              workspace=None, stream=None):
    """Y = act(X·W + bias) + residual, fused into the product. X [M, K], W [K, N],
    bias [N], residual [M, N], all float32 or all bfloat16. gated: W [K, 2N] and
    bias [2N] hold a gate and an up half, Y = act(gate)·up + residual. P: a
    tensor [M, N] ([M, 2N]) that receives the pre-activations for the gradients.
    Y: the output, in the operands' type unless given in float32; it may be
    the residual itself."""
    import torch
    _gpu(X, "X", 2)
    _gpu(W, "W", 2)
    (M, K), wide = X.shape, W.shape[1]
    N = wide // 2 if gated else wide
    if gated and wide % 2:
        raise ValueError("a gated W has an even number of columns")
    dt = _type(X, "X")
    if Y is None:
        Y = _empty((M, N), X.dtype, X.device, stream)
    x, ldx = _tensor(X, "X", X, (M, K))
    w, ldw = _tensor(W, "W", X, (K, wide))
    b = _one(bias, "bias", X, (wide,))
    r, ldr = _pair(residual, "residual", X, (M, N))
    out = _result_type(Y, "Y", X)
    y, ldy = _tensor(Y, "Y", X, (M, N), Y.dtype)
    p, ldp = _pair(P, "P", X, (M, wide))
    _call("gt_linear", gt_linear_args(M, N, K, dt, _act(act, gated), out, 0, x, ldx, w, ldw, b, r,
                                      ldr, y, ldy, p, ldp), X, workspace, stream)
    return Y


def gt_linear_backward(dY, X, W, P=None, act="none", gated=False, bias=True, dX=None, dW=None,
                       db=None, need=("dX", "dW"), workspace=None, stream=None):
    """(dX, dW, db) of gt_linear from dY [M, N] and the P it kept (not needed for act
    "none" without gate). dW in W's type unless given in float32; db float32, None
    unless bias. need: which of dX and dW are wanted. The residual's gradient is
    dY itself."""
    import torch
    _gpu(dY, "dY", 2)
    _gpu(X, "X", 2)
    _gpu(W, "W", 2)
    (M, K), wide = X.shape, W.shape[1]
    N = wide // 2 if gated else wide
    if gated and wide % 2:
        raise ValueError("a gated W has an even number of columns")
    dt, code = _type(X, "X"), _act(act, gated)
    if code and P is None:
        raise ValueError("the gradient of the activation needs P")
    if dX is None and "dX" in need:
        dX = _empty((M, K), X.dtype, X.device, stream)
    if dW is None and "dW" in need:
        dW = _empty((K, wide), W.dtype, W.device, stream)
    if db is None and bias:
        db = _empty((wide,), torch.float32, X.device, stream)
    dy, lddy = _tensor(dY, "dY", X, (M, N))
    x, ldx = _tensor(X, "X", X, (M, K))
    w, ldw = _tensor(W, "W", X, (K, wide))
    p, ldp = _pair(P if code else None, "P", X, (M, wide))
    dx, lddx = _pair(dX, "dX", X, (M, K))
    dwt = F32 if dW is None else _result_type(dW, "dW", W)
    dw, lddw = _pair(dW, "dW", X, (K, wide), None if dW is None else dW.dtype)
    _call("gt_linear_backward",
          gt_linear_grad_args(M, N, K, dt, code, dwt, 0, dy, lddy, x, ldx, w, ldw, p, ldp, dx, lddx,
                              dw, lddw, _one(db, "db", X, (wide,), torch.float32)),
          X, workspace, stream)
    return dX, dW, db


def gt_route(logits, k, bias=None, score="softmax", groups=1, keep=1, renormalise=True, scale=1.0,
             workspace=None, stream=None) -> Route:
    """The k experts of every token by logit + bias, their weights and the lists of
    the experts' rows. logits [T, E] float32 or bfloat16; bias [E] float32,
    for the choice only. The choice is by logit + bias, not by score + bias: a bias
    trained for scores chooses other experts here, and so do groups ranked by
    scores. With groups > 1 the choice is among the `keep` groups of
    E/groups experts whose two largest keys have the largest sum. weights: scale
    times the softmax over the logits or the sigmoid of each, divided by the sum over
    the chosen if renormalise."""
    import torch
    _gpu(logits, "logits", 2)
    T, E = logits.shape
    dt = _type(logits, "logits")
    if score not in SCORES:
        raise ValueError(f"unknown score {score!r}: one of {', '.join(SCORES)}")
    x, ldl = _tensor(logits, "logits", logits, (T, E))
    b = _one(bias, "bias", logits, (E,), torch.float32)
    k = int(k)
    if not 1 <= k <= E:
        raise ValueError(f"k is {k}, with {E} experts")
    n = T * k
    dev = logits.device
    weights = _empty((T, k), torch.float32, dev, stream)
    experts, place, order, offsets = _empty((3 * n + E + 1,), torch.int32, dev, stream).split((n, n, n, E + 1))
    experts, place = experts.view(T, k), place.view(T, k)
    _call("gt_route", gt_route_args(T, E, k, groups, keep, dt, SCORES[score], int(bool(renormalise)),
                                    scale, x, ldl, b, weights.data_ptr(), experts.data_ptr(),
                                    offsets.data_ptr(), order.data_ptr(), place.data_ptr()),
          logits, workspace, stream)
    return Route(weights, experts, offsets, order, place)


def gt_route_backward(dweights, logits, experts, score="softmax", renormalise=True, scale=1.0,
                      dlogits=None, stream=None):
    """The logits' gradient [T, E], in their type, from dweights [T, k] and the
    experts gt_route chose."""
    import torch
    _gpu(logits, "logits", 2)
    _gpu(experts, "experts", 2)
    T, E = logits.shape
    k = experts.shape[1]
    if score not in SCORES:
        raise ValueError(f"unknown score {score!r}: one of {', '.join(SCORES)}")
    if dlogits is None:
        dlogits = _empty((T, E), logits.dtype, logits.device, stream)
    x, ldl = _tensor(logits, "logits", logits, (T, E))
    d, lddl = _tensor(dlogits, "dlogits", logits, (T, E))
    _call("gt_route_backward",
          gt_route_grad_args(T, E, k, _type(logits, "logits"), SCORES[score], int(bool(renormalise)),
                             scale, x, ldl, _whole(experts, "experts", logits, (T, k), torch.int32),
                             _whole(dweights, "dweights", logits, (T, k), torch.float32), d, lddl),
          logits, None, stream)
    return dlogits


def _lists(route, like, T):
    import torch
    weights, experts, offsets, order, place = route
    _gpu(weights, "weights", 2)
    k, E = weights.shape[1], offsets.shape[0] - 1
    return E, k, (_whole(weights, "weights", like, (T, k), torch.float32),
                  _whole(offsets, "offsets", like, (E + 1,), torch.int32),
                  _whole(order, "order", like, (T * k,), torch.int32),
                  _whole(place, "place", like, (T, k), torch.int32))


def _stack(W, name, like, shape):
    """A stack of matrices with contiguous rows: pointer, row stride, matrix stride."""
    p, ld = _tensor(W, name, like, shape)
    return p, ld, W.stride(0) if shape[0] > 1 else ld * shape[1]


def _experts_shapes(X, W1, W2, gated):
    _gpu(X, "X", 2)
    _gpu(W1, "W1", 3)
    _gpu(W2, "W2", 3)
    (T, D), wide = X.shape, W1.shape[2]
    if gated and wide % 2:
        raise ValueError("a gated W1 has an even number of columns")
    return T, D, wide // 2 if gated else wide, wide


def gt_experts(X, route, W1, W2, b1=None, b2=None, residual=None, act="silu", gated=False, Y=None,
               P=None, workspace=None, stream=None):
    """Y[t] = residual[t] + Σ_s weights[t, s]·(act(X[t]·W1[e] + b1[e])·W2[e] + b2[e]) with
    e = route.experts[t, s]. X [T, D], W1 [E, D, H] ([E, D, 2H] gated), W2 [E, H, D],
    b1 [E, H] ([E, 2H]), b2 [E, D]. P: a tensor [T·k, H] ([T·k, 2H]) that receives the
    pre-activations of the experts' rows for the gradients."""
    import torch
    T, D, H, wide = _experts_shapes(X, W1, W2, gated)
    E, k, (weights, offsets, order, place) = _lists(route, X, T)
    if Y is None:
        Y = _empty((T, D), X.dtype, X.device, stream)
    x, ldx = _tensor(X, "X", X, (T, D))
    r, ldr = _pair(residual, "residual", X, (T, D))
    y, ldy = _tensor(Y, "Y", X, (T, D))
    p, ldp = _pair(P, "P", X, (T * k, wide))
    _call("gt_experts",
          gt_experts_args(T, D, H, E, k, _type(X, "X"), _act(act, gated), x, ldx,
                          *_stack(W1, "W1", X, (E, D, wide)), *_stack(W2, "W2", X, (E, H, D)),
                          _one(b1, "b1", X, (E, wide)), _one(b2, "b2", X, (E, D)), r, ldr, y, ldy,
                          p, ldp, weights, offsets, order, place), X, workspace, stream)
    return Y


def gt_experts_backward(dY, X, route, W1, W2, P, b2=None, act="silu", gated=False, bias=True,
                        need=("dX", "dW1", "dW2", "dweights"), workspace=None,
                        stream=None) -> ExpertGrads:
    """The gradients of gt_experts from dY [T, D] and the P it kept: dX, dW1 and dW2 in
    the operands' type, db1, db2 (None unless bias) and dweights [T, k] in float32.
    b2: as given to gt_experts. need: which of dX, dW1, dW2 and dweights are
    wanted. The residual's gradient is dY itself."""
    import torch
    T, D, H, wide = _experts_shapes(X, W1, W2, gated)
    E, k, (weights, offsets, order, place) = _lists(route, X, T)
    dev, f32 = X.device, torch.float32

    def new(name, dtype, *shape):
        return _empty(shape, dtype, dev, stream) if name in need else None

    g = ExpertGrads(new("dX", X.dtype, T, D), new("dW1", X.dtype, E, D, wide),
                    new("dW2", X.dtype, E, H, D),
                    _empty((E, wide), f32, dev, stream) if bias else None,
                    _empty((E, D), f32, dev, stream) if bias else None,
                    new("dweights", f32, T, k))
    dy, lddy = _tensor(dY, "dY", X, (T, D))
    x, ldx = _tensor(X, "X", X, (T, D))
    p, ldp = _tensor(P, "P", X, (T * k, wide))
    ptr = [None if t is None else t.data_ptr() for t in g]
    _call("gt_experts_backward",
          gt_experts_grad_args(T, D, H, E, k, _type(X, "X"), _act(act, gated), dy, lddy, x, ldx,
                               *_stack(W1, "W1", X, (E, D, wide)), *_stack(W2, "W2", X, (E, H, D)),
                               _one(b2, "b2", X, (E, D)), p, ldp, weights, offsets, order, place,
                               ptr[0], D, *ptr[1:]), X, workspace, stream)
    return g
