"""The operators around layers in 8-bit floating point this framework is measured on.

Four operators, which a layer with 8-bit operands runs one after the other:

  norm           Y = (X - mean)·rstd·w + b over each row, and in training the rows' mean and rstd; or
                 Y in 8 bits at once, as the next layer's product takes it
  norm_backward  g = dY·w, dX = rstd·(g - mean(g) - xh·mean(g·xh)) + R with xh = (X - mean)·rstd,
                 dw = Σ rows of dY·xh, db = Σ rows of dY
  quantise       8-bit codes with one scale for each 128 values of a row, or for each square of
                 128×128 values, and the same of the transpose: scale = largest/(the type's largest),
                 code = X/scale rounded to nearest even
  linear_fp8     Y = act(X·Wᵀ + b) + R of such codes, X·Wᵀ = Σ over blocks of 128 of
                 (scale of X)·(scale of W)·Σ codes·codes

`run` computes them in plain 32-bit torch operations or, where `own` is set, by the framework's
calls; `exact` computes them in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
FP8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}
SIZE = {"f32": 4, "bf16": 2}
BLOCK = 128
EPS = 1e-5
# passes are priced at these rates (bytes/s, operations/s) when a drawn case is held to the listed
PRICE = {"bytes": 5e12, "flops": 1e15}


def _norm(name, dtype, M, N, wtype=None, train=False, code="none", pow2=False):
    return {"name": name, "op": "norm", "dtype": dtype, "M": M, "N": N, "wtype": wtype or dtype,
            "train": train, "code": code, "pow2": pow2}


def _norm_backward(name, dtype, M, N, wtype=None, residual=False):
    return {"name": name, "op": "norm_backward", "dtype": dtype, "M": M, "N": N,
            "wtype": wtype or dtype, "residual": residual}


def _quantise(name, dtype, M, N, block, code="e4m3", transposed=False, pow2=False):
    return {"name": name, "op": "quantise", "dtype": dtype, "M": M, "N": N, "block": block,
            "code": code, "transposed": transposed, "pow2": pow2}


def _linear(name, M, N, K, dtype="bf16", out="", wblock="square", xcode="e4m3", wcode="e4m3",
            act="none", gated=False, bias=False, residual=False):
    return {"name": name, "op": "linear_fp8", "dtype": dtype, "out": out or dtype, "M": M, "N": N,
            "K": K, "wblock": wblock, "xcode": xcode, "wcode": wcode, "act": act, "gated": gated,
            "bias": bias, "residual": residual}


def listed():
    return [
        # the norm of one generated token: latency
        _norm("norm_token_bf16", "bf16", 1, 4096),
        # the norm of a training batch, its statistics kept, parameters in fp32
        _norm("norm_train_bf16", "bf16", 16384, 4096, wtype="f32", train=True),
        # the norm in front of a layer with 8-bit operands: its rows leave as codes
        _norm("norm_codes_bf16", "bf16", 4096, 4096, train=True, code="e4m3"),
        # the gradients of a training batch's norm, joined with the residual path's
        _norm_backward("norm_backward_bf16", "bf16", 16384, 4096, wtype="f32", residual=True),
        # odd extents in fp32: no row but the first begins on a 16-byte boundary
        _norm_backward("norm_backward_f32", "f32", 999, 1021),
        # the gradient of a wide layer's rows, for the input's and for the weight's product
        _quantise("quantise_gradient_bf16", "bf16", 4096, 11008, "row", code="e5m2", transposed=True),
        # odd-sized fp32 weights after an optimiser's step, in both layouts
        _quantise("quantise_weight_f32", "f32", 2623, 3457, "square", transposed=True, pow2=True),
        # the gate and up products of one generated token: reads the weights and little else
        _linear("linear_token", 1, 11008, 4096, act="silu", gated=True),
        # a batch of 64 against a square weight, added to its residual
        _linear("linear_batch", 64, 4096, 4096, bias=True, residual=True),
        # an MLP's up-projection over 4096 tokens
        _linear("linear_mlp", 4096, 11008, 4096, bias=True),
        # the weight's gradient of a square layer over 4096 tokens: scales along both operands' rows
        _linear("linear_weight_gradient", 4096, 4096, 4096, out="f32", wblock="row", wcode="e5m2"),
        # odd extents everywhere
        _linear("linear_ragged", 1999, 2623, 3457, act="gelu", bias=True, residual=True),
    ]


def _size(rng, lo, hi):
    """An extent in [lo, hi], spread over its logarithm: a third powers of two, a third multiples
    of 8, a third any number."""
    v = 2.0 ** rng.uniform(math.log2(lo), math.log2(hi))
    kind = rng.randrange(3)
    n = 2 ** round(math.log2(v)) if kind == 0 else 8 * round(v / 8) if kind == 1 else round(v)
    return min(hi, max(lo, n))


def _cost(case):
    w = work(case)
    return w["bytes"] / PRICE["bytes"] + w["flops"] / PRICE["flops"]


def _drawn(rng):
    op = rng.choice(("norm", "norm_backward", "quantise", "linear_fp8", "linear_fp8"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    code = rng.choice(("e4m3", "e4m3", "e5m2"))
    one, two, three, four = (rng.random() < 0.5 for _ in range(4))
    if op == "linear_fp8":
        return _linear("", _size(rng, 1, 4096), _size(rng, 64, 11008), _size(rng, 64, 4096), dtype,
                       rng.choice((dtype, "f32")), rng.choice(("square", "square", "row")), code,
                       rng.choice(("e4m3", "e4m3", "e5m2")),
                       rng.choice(("none", "none", "relu", "gelu", "silu")), one, two, three)
    M, N = _size(rng, 1, 16384), _size(rng, 64, 16384)
    wtype = rng.choice((dtype, "f32"))
    if op == "norm":
        return _norm("", dtype, M, N, wtype, one, code if two else "none", two and three)
    if op == "norm_backward":
        return _norm_backward("", dtype, M, N, wtype, one)
    return _quantise("", dtype, M, N, rng.choice(("row", "square")), code, one, two)


def draw(rng):
    """Another case of the listed ranges (no name) that costs no more than the largest listed one."""
    most = max(_cost(c) for c in listed())
    while True:
        c = _drawn(rng)
        if _cost(c) <= most:
            del c["name"]
            return c


# --------------------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------------------

def _device():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


def _draws(seed):
    dev = _device()
    gen = torch.Generator(device=dev).manual_seed(seed)

    def normal(dtype, *shape, std=1.0):
        return torch.randn(*shape, generator=gen, device=dev).mul_(std).to(TYPES[dtype])

    return normal


def _rows(normal, dtype, M, N):
    """Activations: columns of unequal size, some of them far larger than the others, off centre."""
    size = torch.exp(normal("f32", N, std=0.7))
    return (normal("f32", M, N) * size + 0.3 * normal("f32", N)).to(TYPES[dtype])


def _blocks(n):
    return -(-n // BLOCK)


def _codes(X, block, code, pow2=False):
    """Codes and scales of a matrix in 32 bits."""
    M, N = X.shape
    b = _blocks(N)
    size = torch.zeros(M, b * BLOCK, device=X.device)
    size[:, :N] = X.abs()
    most = size.view(M, b, BLOCK).amax(2)
    if block == "square":
        rows = torch.zeros(_blocks(M) * BLOCK, b, device=X.device)
        rows[:M] = most
        most = rows.view(-1, BLOCK, b).amax(1)
    scale = (most / LARGEST[code]).clamp(min=2.0 ** -126)
    if pow2:   # the next power of two
        part, exponent = torch.frexp(scale)
        scale = torch.ldexp(torch.ones_like(scale), torch.where(part == 0.5, exponent - 1, exponent))
    scale = torch.where(most == 0, 1.0, scale)
    back = (1.0 / scale).repeat_interleave(BLOCK, dim=1)[:, :N]
    if block == "square":
        back = back.repeat_interleave(BLOCK, dim=0)[:M]
    return (X * back).to(FP8[code]), scale


def _padded(q):
    """The same codes in rows of whole 16-byte chunks."""
    M, K = q.shape
    wide = torch.zeros(M, -(-K // 16) * 16, dtype=torch.uint8, device=q.device)
    wide[:, :K] = q.view(torch.uint8)
    return wide.view(q.dtype)[:, :K]


def prepare(case, seed):
    normal = _draws(seed)
    op, dt = case["op"], case["dtype"]
    s = {"case": case}
    if op == "linear_fp8":
        M, N, K = case["M"], case["N"], case["K"]
        wide = N * (2 if case["gated"] else 1)
        q, sc = _codes(_rows(normal, "f32", M, K), "row", case["xcode"])
        s["X"], s["sx"] = _padded(q), sc
        q, sc = _codes(normal("f32", wide, K, std=K ** -0.5), case["wblock"], case["wcode"])
        s["W"], s["sw"] = _padded(q), sc
        s["bias"] = normal(dt, wide, std=0.1) if case["bias"] else None
        s["residual"] = normal(dt, M, N) if case["residual"] else None
        return s
    M, N = case["M"], case["N"]
    s["X"] = _rows(normal, dt, M, N)
    if op == "quantise":
        return s
    s["w"] = (1 + normal("f32", N, std=0.2)).to(TYPES[case["wtype"]])
    if op == "norm":
        s["b"] = normal(case["wtype"], N, std=0.2)
        return s
    x = s["X"].double()   # the statistics that the forward pass left
    s["mean"] = x.mean(1).float()
    s["rstd"] = (x.var(1, unbiased=False) + EPS).rsqrt().float()
    s["dY"] = normal(dt, M, N)
    s["R"] = normal(dt, M, N) if case["residual"] else None
    return s


# --------------------------------------------------------------------------------------------------
# the plain forms, in 32 bits
# --------------------------------------------------------------------------------------------------

def _plain_norm(s, c):
    x = s["X"].float()
    mean = x.sum(1, keepdim=True) / c["N"]
    d = x - mean
    rstd = 1 / torch.sqrt((d * d).sum(1, keepdim=True) / c["N"] + EPS)
    Y = d * rstd * s["w"].float() + s["b"].float()
    out = {"mean": mean.squeeze(1), "rstd": rstd.squeeze(1)} if c["train"] else {}
    if c["code"] == "none":
        return {**out, "Y": Y.to(TYPES[c["dtype"]])}
    out["codes"], out["scales"] = _codes(Y, "row", c["code"], c["pow2"])
    return out


def _plain_norm_backward(s, c):
    rstd = s["rstd"].unsqueeze(1)
    xh = (s["X"].float() - s["mean"].unsqueeze(1)) * rstd
    dY = s["dY"].float()
    g = dY * s["w"].float()
    dX = rstd * (g - g.sum(1, keepdim=True) / c["N"] - xh * ((g * xh).sum(1, keepdim=True) / c["N"]))
    if s["R"] is not None:
        dX = dX + s["R"].float()
    return {"dX": dX.to(TYPES[c["dtype"]]), "dw": (dY * xh).sum(0), "db": dY.sum(0)}


def _plain_quantise(s, c):
    X = s["X"].float()
    q, sc = _codes(X, c["block"], c["code"], c["pow2"])
    out = {"codes": q, "scales": sc}
    if c["transposed"]:
        out["tcodes"], out["tscales"] = _codes(X.T.contiguous(), c["block"], c["code"], c["pow2"])
    return out


def _spread(scale, rows, cols, block):
    """A scale for each value."""
    s = scale.repeat_interleave(BLOCK, dim=1)[:, :cols]
    return s.repeat_interleave(BLOCK, dim=0)[:rows] if block == "square" else s


def _act(x, act):
    if act == "relu":
        return torch.where(x > 0, x, 0.0)
    if act == "gelu":
        return 0.5 * x * (1 + torch.erf(x * 0.5 ** 0.5))
    if act == "silu":
        return x / (1 + torch.exp(-x))
    return x


def _plain_linear(s, c):
    wide = c["N"] * (2 if c["gated"] else 1)
    X = s["X"].float() * _spread(s["sx"], c["M"], c["K"], "row")
    W = s["W"].float() * _spread(s["sw"], wide, c["K"], c["wblock"])
    P = X @ W.T
    if s["bias"] is not None:
        P = P + s["bias"].float()
    Y = _act(P[:, :c["N"]], c["act"]) * P[:, c["N"]:] if c["gated"] else _act(P, c["act"])
    if s["residual"] is not None:
        Y = Y + s["residual"].float()
    return {"Y": Y.to(TYPES[c["out"]])}


# --------------------------------------------------------------------------------------------------
# the framework's calls
# --------------------------------------------------------------------------------------------------

def _own(s, c):
    from paper_1909_10616_amd import layers
    op, X = c["op"], s["X"]
    if op == "linear_fp8":
        Y = torch.empty(c["M"], c["N"], dtype=TYPES[c["out"]], device=X.device)
        layers.gt_linear_fp8(layers.Codes(X, s["sx"]), layers.Codes(s["W"], s["sw"]), bias=s["bias"],
                             residual=s["residual"], act=c["act"], gated=c["gated"], Y=Y)
        return {"Y": Y}
    if op == "quantise":
        need = ("codes", "transposed") if c["transposed"] else ("codes",)
        codes, transposed = layers.gt_quantise(X, block=c["block"], code=c["code"], pow2=c["pow2"],
                                               need=need)
        out = {"codes": codes.values, "scales": codes.scales}
        if c["transposed"]:
            out["tcodes"], out["tscales"] = transposed
        return out
    if op == "norm":
        out = {}
        if c["train"]:
            out["mean"], out["rstd"] = torch.empty(2, c["M"], device=X.device)
        if c["code"] == "none":
            out["Y"] = layers.gt_norm(X, s["w"], s["b"], eps=EPS, mean=out.get("mean"),
                                      rstd=out.get("rstd"))
        else:
            out["codes"], out["scales"] = layers.gt_norm_fp8(
                X, s["w"], s["b"], eps=EPS, code=c["code"], pow2=c["pow2"], mean=out.get("mean"),
                rstd=out.get("rstd"))
        return out
    dX, dw, db = layers.gt_norm_backward(s["dY"], X, s["mean"], s["rstd"], weight=s["w"],
                                         residual=s["R"])
    return {"dX": dX, "dw": dw, "db": db}


PLAIN = {"norm": _plain_norm, "norm_backward": _plain_norm_backward, "quantise": _plain_quantise,
         "linear_fp8": _plain_linear}


def run(state):
    case = state["case"]
    return _own(state, case) if own else PLAIN[case["op"]](state, case)


# --------------------------------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------------------------------

def _scales(rows, cols, block):
    return (_blocks(rows) if block == "square" else rows) * _blocks(cols) * 4


def work(case):
    op, size, M, N = case["op"], SIZE[case["dtype"]], case["M"], case["N"]
    if op == "linear_fp8":
        K = case["K"]
        wide = N * (2 if case["gated"] else 1)
        nbytes = M * K + wide * K + _scales(M, K, "row") + _scales(wide, K, case["wblock"])
        nbytes += (wide * size if case["bias"] else 0) + (M * N * size if case["residual"] else 0)
        return {"bytes": nbytes + M * N * SIZE[case["out"]], "flops": 2 * M * wide * K}
    if op == "quantise":
        each = M * N + _scales(M, N, case["block"])
        nbytes = M * N * size + each
        if case["transposed"]:
            nbytes += M * N + _scales(N, M, case["block"])
        return {"bytes": nbytes, "flops": M * N * (4 if case["transposed"] else 2)}
    if op == "norm":
        out = M * N * size if case["code"] == "none" else M * N + _scales(M, N, "row")
        nbytes = M * N * size + out + 2 * N * SIZE[case["wtype"]] + (8 * M if case["train"] else 0)
        return {"bytes": nbytes, "flops": 8 * M * N}
    nbytes = M * N * size * (4 if case["residual"] else 3) + 8 * M + N * SIZE[case["wtype"]] + 8 * N
    return {"bytes": nbytes, "flops": 14 * M * N}


# --------------------------------------------------------------------------------------------------
# the definitions, in 64 bits
# --------------------------------------------------------------------------------------------------

def _exact_codes(X, case, block):
    """Codes by division in 64 bits by the scale that is stored."""
    top = LARGEST[case["code"]]
    out = torch.zeros_like(X)
    M, N = X.shape
    step = BLOCK if block == "square" else M
    scales = []
    for r in range(0, M, step):
        line = []
        for c in range(0, N, BLOCK):
            part = X[r:r + step, c:c + BLOCK]
            most = part.abs().amax() if block == "square" else part.abs().amax(1, keepdim=True)
            scale = most / top
            if case["pow2"]:
                scale = torch.exp2(torch.ceil(torch.log2(scale)))
            scale = torch.where(most > 0, scale.clamp(min=2.0 ** -126), 1.0)
            out[r:r + step, c:c + BLOCK] = part / scale
            line.append(scale.reshape(-1, 1))
        scales.append(torch.cat(line, dim=1))
    return out.to(FP8[case["code"]]), torch.cat(scales, dim=0)


def exact(case, seed):
    s = {n: v.double() if isinstance(v, torch.Tensor) else v for n, v in prepare(case, seed).items()}
    op, X = case["op"], s["X"]
    if op == "linear_fp8":
        wide = s["W"].shape[0]
        x = torch.repeat_interleave(s["sx"], BLOCK, dim=1).narrow(1, 0, case["K"])
        w = torch.repeat_interleave(s["sw"], BLOCK, dim=1).narrow(1, 0, case["K"])
        if case["wblock"] == "square":
            w = torch.repeat_interleave(w, BLOCK, dim=0).narrow(0, 0, wide)
        P = torch.mm(X * x, torch.mul(s["W"], w).t())
        P += 0 if s["bias"] is None else s["bias"]
        gate, up = P.chunk(2, dim=1) if case["gated"] else (P, 1.0)
        value = {"none": lambda v: v, "relu": lambda v: v.clamp(min=0), "silu": torch.nn.functional.silu,
                 "gelu": lambda v: v * torch.special.ndtr(v)}[case["act"]]
        Y = value(gate) * up
        return {"Y": Y if s["residual"] is None else Y + s["residual"]}
    if op == "quantise":
        out = dict(zip(("codes", "scales"), _exact_codes(X, case, case["block"])))
        if case["transposed"]:
            out.update(zip(("tcodes", "tscales"), _exact_codes(X.t(), case, case["block"])))
        return out
    if op == "norm":
        mean, var = X.mean(dim=1), X.var(dim=1, unbiased=False)
        rstd = torch.rsqrt(var + EPS)
        Y = torch.addcmul(s["b"], (X - mean[:, None]) * rstd[:, None], s["w"])
        out = {"mean": mean, "rstd": rstd} if case["train"] else {}
        if case["code"] == "none":
            return {**out, "Y": Y}
        return {**out, **dict(zip(("codes", "scales"), _exact_codes(Y, case, "row")))}
    xh = (X - s["mean"][:, None]) * s["rstd"][:, None]
    g = s["dY"] * s["w"]
    # the part of g that is neither constant along the row nor along xh
    dX = g - g.mean(dim=1, keepdim=True) - xh * (xh * g).mean(dim=1, keepdim=True)
    dX = dX * s["rstd"][:, None]
    return {"dX": dX if s["R"] is None else dX + s["R"],
            "dw": torch.einsum("mn,mn->n", s["dY"], xh), "db": s["dY"].sum(dim=0)}
