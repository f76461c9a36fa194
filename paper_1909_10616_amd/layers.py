"""Layer operators of libgemmtune (include/gemmtune_layers.h), same names as the
C ABI: perceptron layers with their epilogue, their gradients, the routing of
tokens to experts, layers of experts, and layers in 8-bit floating point with the
norm before them.

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
CODES = {"e4m3": 0, "e5m2": 1}
BLOCKS = {"row": 1, "square": 128}   # rows that share a scale

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


class gt_quantise_args(ctypes.Structure):
    _fields_ = _fields("l:M N;i:dtype code block pow2;p:X;l:ldx;p:Q;l:ldq;p:S;l:lds;p:Qt;l:ldqt;p:St;l:ldst")


class gt_linear_fp8_args(ctypes.Structure):
    _fields_ = _fields("l:M N K;i:dtype act out_dtype xcode wcode xblock wblock exact;p:X;l:ldx;p:sx;"
                       "l:ldsx;p:W;l:ldw;p:sw;l:ldsw;p:bias R;l:ldr;p:Y;l:ldy")


class gt_norm_args(ctypes.Structure):
    _fields_ = _fields("l:M N;i:dtype wtype code pow2;f:eps;i:reserved;p:X;l:ldx;p:w b Y;l:ldy;p:mean rstd "
                       "Q;l:ldq;p:S;l:lds")


class gt_norm_grad_args(ctypes.Structure):
    _fields_ = _fields("l:M N;i:dtype wtype;p:dY;l:lddy;p:X;l:ldx;p:w mean rstd R;l:ldr;p:dX;l:lddx;p:dw db")


# entry point → its argument structure; those with a scratch have a _workspace
EXPORTS = {"gt_linear": gt_linear_args, "gt_linear_backward": gt_linear_grad_args,
           "gt_route": gt_route_args, "gt_route_backward": gt_route_grad_args,
           "gt_experts": gt_experts_args, "gt_experts_backward": gt_experts_grad_args,
           "gt_quantise": gt_quantise_args, "gt_linear_fp8": gt_linear_fp8_args,
           "gt_norm": gt_norm_args, "gt_norm_backward": gt_norm_grad_args}
NO_SCRATCH = ("gt_route_backward", "gt_quantise", "gt_norm")


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


class Codes(typing.NamedTuple):
    """A matrix in 8-bit floating point: it stands for values·scales, a scale for 128 values
    of a row, or for a square of 128×128."""
    values: typing.Any    # float8_e4m3fn or float8_e5m2 [R, C]
    scales: typing.Any    # float32 [R, ceil(C/128)], or [ceil(R/128), ceil(C/128)]


class Quantised(typing.NamedTuple):
    codes: typing.Any        # Codes of X, None if not wanted
    transposed: typing.Any   # Codes of its transpose


class NormGrads(typing.NamedTuple):
    dX: typing.Any
    dweight: typing.Any
    dbias: typing.Any


_NORM_GRADS = frozenset(NormGrads._fields)


_lib = None
_calls = {}   # entry point → its function and its scratch query (None: no scratch)


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
                _calls[name] = f, None
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
    if t.get_device() != like.get_device():
        raise ValueError(f"{name} must be a GPU tensor on {like.device}")
    have = t.shape
    if have != shape:
        raise ValueError(f"{name} has shape {tuple(have)}, not {tuple(shape)}")
    st = t.stride()
    n = len(st)
    if n == 2 and st[1] == 1 and st[0] >= have[1] > 0:   # (nearly every call)
        return t.data_ptr(), st[0]
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
    if _lib is None:
        lib()
    device = like.get_device()
    if device == torch._C._cuda_getDevice():
        # (the current stream's handle alone, as _stream gives it)
        on = torch._C._cuda_getCurrentRawStream(device) if stream is None else _stream(stream)
        _launch(name, a, like, workspace, stream, on)
        return
    with torch.cuda.device(device):
        _launch(name, a, like, workspace, stream, _stream(stream))


def _launch(name, a, like, workspace, stream, on):
    run, query = _calls[name]
    ref = ctypes.byref(a)
    if query is None:
        rc = run(ref, on)
    else:
        need = _i64()
        _check(query(ref, ctypes.byref(need)), name)
        n = need.value
        if n == 0:
            rc = run(ref, None, 0, on)
        else:
            if workspace is None:
                import torch
                workspace = _empty((n,), torch.uint8, like.device, stream)
            elif workspace.device != like.device or not workspace.is_contiguous():
                raise ValueError("workspace must be contiguous, on the operands' device")
            rc = run(ref, workspace.data_ptr(), workspace.numel() * workspace.element_size(), on)
    if rc != 0:
        _check(rc, name)


def _empty(shape, dtype, device, stream, ld=None):
    """Memory for the stream the call runs on (PyTorch's allocator gives memory that is
    free in the order of one stream); ld: elements between rows."""
    import torch
    if stream is None:   # (strides given: a third of a microsecond less than torch.empty)
        n = len(shape)
        if n == 2:
            return torch.empty_strided(shape, (ld or shape[1] or 1, 1), dtype=dtype, device=device)
        if n == 1:
            return torch.empty_strided(shape, (1,), dtype=dtype, device=device)
        return torch.empty(shape, dtype=dtype, device=device)
    if not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(int(stream), device=device)
    with torch.cuda.stream(stream):
        return _empty(shape, dtype, device, None, ld)


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


# ---- layers in 8-bit floating point

def _blocks(n):
    return (n + 127) // 128


def _code(code):
    if code not in CODES:
        raise ValueError(f"unknown code {code!r}: one of {', '.join(CODES)}")
    return CODES[code]


def _code_of(t, name):
    import torch
    if t.dtype is torch.float8_e4m3fn:
        return CODES["e4m3"]
    if t.dtype is torch.float8_e5m2:
        return CODES["e5m2"]
    raise ValueError(f"{name} must be float8_e4m3fn or float8_e5m2")


def _new_codes(rows, cols, code, block, device, stream):
    """Codes to be filled: rows of whole 16-byte chunks, which the products read fastest."""
    import torch
    dtype = torch.float8_e4m3fn if code == CODES["e4m3"] else torch.float8_e5m2
    return Codes(_empty((rows, cols), dtype, device, stream, (cols + 15) // 16 * 16),
                 _empty((rows if block == 1 else _blocks(rows), _blocks(cols)), torch.float32, device, stream))


def _codes(c, name, like, shape):
    """A matrix of codes: its type, the rows that share a scale, both pointers and row strides."""
    import torch
    values, scales = c
    code = _code_of(values, name)
    q, ldq = _tensor(values, name, like, shape, values.dtype)
    rows, cols = shape
    block = 1 if scales.dim() == 2 and scales.shape[0] == rows else 128
    s, lds = _tensor(scales, f"the scales of {name}", like, (rows if block == 1 else _blocks(rows), _blocks(cols)),
                     torch.float32)
    return code, block, q, ldq, s, lds


def gt_quantise(X, block="row", code="e4m3", pow2=False, need=("codes",), stream=None) -> Quantised:
    """8-bit codes of X [M, N] with a scale for each 128 values of a row (block "row") or each
    square of 128×128 ("square"). A scale is the block's largest magnitude over the type's (448;
    57344 for code "e5m2"), with pow2 the next power of two. need: "codes" of X, and "transposed",
    codes of its transpose with blocks along M, as the products of the gradients take them."""
    _gpu(X, "X", 2)
    M, N = X.shape
    if block not in BLOCKS:
        raise ValueError(f"unknown block {block!r}: one of {', '.join(BLOCKS)}")
    need = (need,) if isinstance(need, str) else tuple(need)
    if not need or set(need) - {"codes", "transposed"}:
        raise ValueError('need is "codes", "transposed" or both')
    c, b = _code(code), BLOCKS[block]
    x, ldx = _tensor(X, "X", X, (M, N))
    dt = _type(X, "X")
    q = _new_codes(M, N, c, b, X.device, stream) if "codes" in need else None
    t = _new_codes(N, M, c, b, X.device, stream) if "transposed" in need else None
    _call("gt_quantise",
          gt_quantise_args(M, N, dt, c, b, int(bool(pow2)), x, ldx, *_places(q), *_places(t)), X, None, stream)
    return Quantised(q, t)


def _places(c):
    if c is None:
        return None, 0, None, 0
    values, scales = c
    return (values.data_ptr(), max(values.stride(0), values.shape[1]), scales.data_ptr(),
            max(scales.stride(0), scales.shape[1]))


def gt_linear_fp8(X, W, bias=None, residual=None, act="none", gated=False, Y=None, workspace=None,
                  stream=None, exact=False):
    """Y = act(X·Wᵀ + bias) + residual of Codes X [M, K] and W [N, K], fused into the product: K
    lies along the rows of both, blocks of 128 of it are summed and scaled in fp32. gated: W [2N, K]
    and bias [2N] hold a gate's rows, then the up's, Y = act(gate)·up + residual. bias and residual
    [M, N] float32 or bfloat16, of one type; Y in that type (bfloat16 without either) unless given,
    in float32 or in theirs; it may be the residual itself. A bfloat16 Y lets the 8-bit matrix instructions
    add a block's products, which keep some 13 bits below the largest of 8; a float32 Y and exact=True
    have them added in fp32, at about half the rate. The gradients are products of
    codes too: dX = gt_linear_fp8(codes of dY, transposed codes of W), dW [N, K] =
    gt_linear_fp8(transposed codes of dY, transposed codes of X)."""
    import torch
    try:
        (like, _), (values, _) = X, W
        wide, K = values.shape
    except (TypeError, ValueError, AttributeError):
        like = None
    if not isinstance(like, torch.Tensor) or isinstance(X, torch.Tensor) or isinstance(W, torch.Tensor):
        raise ValueError("X and W must be Codes of matrices: values and their scales")
    _gpu(like, "X", 2)
    M = like.shape[0]
    N = wide // 2 if gated else wide
    if gated and wide % 2:
        raise ValueError("a gated W has an even number of rows")
    xc, xb, x, ldx, sx, ldsx = _codes(X, "X", like, (M, K))
    wc, wb, w, ldw, sw, ldsw = _codes(W, "W", like, (wide, K))
    typed = bias if bias is not None else residual
    if Y is None:
        Y = _empty((M, N), torch.bfloat16 if typed is None else typed.dtype, like.device, stream)
        y, ldy = Y.data_ptr(), N
    else:
        y, ldy = _tensor(Y, "Y", like, (M, N), Y.dtype)
    typed = Y if typed is None else typed
    dt = _type(typed, "Y" if typed is Y else "bias" if typed is bias else "residual")
    b = _one(bias, "bias", like, (wide,), typed.dtype)
    r, ldr = _pair(residual, "residual", like, (M, N), typed.dtype)
    out = _result_type(Y, "Y", typed)
    _call("gt_linear_fp8",
          gt_linear_fp8_args(M, N, K, dt, _act(act, gated), out, xc, wc, xb, wb, int(bool(exact)), x, ldx, sx, ldsx,
                             w, ldw, sw, ldsw, b, r, ldr, y, ldy), like, workspace, stream)
    return Y


def _norm(X, weight, bias, eps, y, ldy, mean, rstd, codes, code, pow2, stream):
    import torch
    M, N = X.shape
    dt = _type(X, "X")
    eps = float(eps)
    if not 0.0 <= eps < float("inf"):
        raise ValueError(f"eps is {eps}: finite and not negative")
    x, ldx = _tensor(X, "X", X, (M, N))
    typed = weight if weight is not None else bias if bias is not None else X
    wt = _result_type(typed, "weight" if typed is weight else "bias", X)
    w = _one(weight, "weight", X, (N,), typed.dtype)
    b = _one(bias, "bias", X, (N,), typed.dtype)
    _call("gt_norm",
          gt_norm_args(M, N, dt, wt, code, int(bool(pow2)), eps, 0, x, ldx, w, b, y, ldy,
                       _one(mean, "mean", X, (M,), torch.float32), _one(rstd, "rstd", X, (M,), torch.float32),
                       *_places(codes)), X, None, stream)


def gt_norm(X, weight=None, bias=None, eps=1e-5, Y=None, mean=None, rstd=None, stream=None):
    """Layer norm: Y = (X − mean)·rstd·weight + bias over the rows of X [M, N], rstd =
    1/√(variance + eps). weight, bias [N]: in X's type or float32. mean, rstd: float32 tensors
    [M] that receive the rows' statistics for the gradients. Y may be X itself."""
    _gpu(X, "X", 2)
    if Y is None:
        Y = _empty(X.shape, X.dtype, X.device, stream)
        y, ldy = Y.data_ptr(), X.shape[1]
    else:
        y, ldy = _tensor(Y, "Y", X, X.shape)
    _norm(X, weight, bias, eps, y, ldy, mean, rstd, None, 0, False, stream)
    return Y


def gt_norm_fp8(X, weight=None, bias=None, eps=1e-5, code="e4m3", pow2=False, Y=None, mean=None, rstd=None,
                stream=None) -> Codes:
    """gt_norm whose result leaves as Codes with a scale for each 128 values of a row, as
    gt_quantise would give them of the unrounded values: what gt_linear_fp8 takes. Y: a tensor that
    receives the values as well."""
    _gpu(X, "X", 2)
    c = _code(code)
    y, ldy = _pair(Y, "Y", X, X.shape)
    codes = _new_codes(*X.shape, c, 1, X.device, stream)
    _norm(X, weight, bias, eps, y, ldy, mean, rstd, codes, c, pow2, stream)
    return codes


def gt_norm_backward(dY, X, mean, rstd, weight=None, residual=None, bias=True, dX=None,
                     need=("dX", "dweight"), workspace=None, stream=None) -> NormGrads:
    """The gradients of gt_norm from dY [M, N] and the statistics it kept: dX in X's type, dweight
    and dbias (None unless bias) [N] in float32. residual [M, N]: a gradient that reaches X by
    another way, added to dX. dX may be the residual or dY itself. need: which of "dX" and "dweight" are
    wanted; dbias is wanted with bias, or where it is named there. The sums over the columns read X and dY a
    second time or take scratch: of dX alone, need="dX", bias=False leaves them out."""
    import torch
    need = (need,) if isinstance(need, str) else tuple(need)
    if not _NORM_GRADS.issuperset(need):
        raise ValueError('need is "dX", "dweight", "dbias" or several of them')
    _gpu(dY, "dY", 2)
    _gpu(X, "X", 2)
    M, N = X.shape
    dt = _type(X, "X")
    if dX is not None:
        dx, lddx = _tensor(dX, "dX", X, (M, N))
    elif "dX" in need:
        dX = _empty((M, N), X.dtype, X.device, stream)
        dx, lddx = dX.data_ptr(), N
    else:
        dx, lddx = None, 0
    dw = _empty((N,), torch.float32, X.device, stream) if "dweight" in need else None
    db = _empty((N,), torch.float32, X.device, stream) if bias or "dbias" in need else None
    dy, lddy = _tensor(dY, "dY", X, (M, N))
    x, ldx = _tensor(X, "X", X, (M, N))
    wt = dt if weight is None else _result_type(weight, "weight", X)
    w = None if weight is None else _whole(weight, "weight", X, (N,), weight.dtype)
    r, ldr = _pair(residual, "residual", X, (M, N))
    _call("gt_norm_backward",
          gt_norm_grad_args(M, N, dt, wt, dy, lddy, x, ldx, w, _whole(mean, "mean", X, (M,), torch.float32),
                            _whole(rstd, "rstd", X, (M,), torch.float32), r, ldr, dx, lddx,
                            None if dw is None else dw.data_ptr(), None if db is None else db.data_ptr()),
          X, workspace, stream)
    return NormGrads(dX, dw, db)
