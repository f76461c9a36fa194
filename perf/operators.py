"""The layer operators this framework is measured on.

Five operators of perceptron layers, dense and with routed experts:

  linear            Y = act(X·W + b) + R, P = X·W + b kept for training; gated: W holds a gate and
                    an up half, Y = act(P_gate)·P_up + R
  linear_backward   dP = dY·act'(P), dX = dP·Wᵀ, dW = Xᵀ·dP, db = Σ rows of dP
  route             the k experts of every token by the score of logit + bias (within the kept
                    groups), their weights, and the lists that sort the tokens by expert; in
                    training also the gradient of the logits
  experts           Y[t] = R[t] + Σ_s w[t,s]·(act(X[t]·W1[e] + b1[e])·W2[e] + b2[e]), e = expert s of t
  experts_backward  the gradients of X, W1, b1, W2, b2 and w

`run` computes them in plain 32-bit torch operations or, where `own` is set, by the framework's
calls; `exact` computes them in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
# passes are priced at these rates (bytes/s, operations/s) when a drawn case is held to the listed
PRICE = {"bytes": 5e12, "f32": 1e14, "bf16": 1e15}


def _linear(name, dtype, M, N, K, act, gated=False, bias=False, residual=False, train=False):
    return {"name": name, "op": "linear", "dtype": dtype, "M": M, "N": N, "K": K, "act": act,
            "gated": gated, "bias": bias, "residual": residual, "train": train}


def _linear_backward(name, dtype, M, N, K, act, gated=False, bias=False):
    return {"name": name, "op": "linear_backward", "dtype": dtype, "M": M, "N": N, "K": K,
            "act": act, "gated": gated, "bias": bias}


def _route(name, dtype, T, E, k, score, groups=1, keep=1, bias=False, renormalise=True, scale=1.0,
           train=False, shut=0.0):
    return {"name": name, "op": "route", "dtype": dtype, "T": T, "E": E, "k": k, "score": score,
            "groups": groups, "keep": keep, "bias": bias, "renormalise": renormalise,
            "scale": scale, "train": train, "shut": shut}


def _experts(name, op, dtype, T, E, k, D, H, act, gated, bias=False, residual=False, train=False):
    return {"name": name, "op": op, "dtype": dtype, "T": T, "E": E, "k": k, "D": D, "H": H,
            "act": act, "gated": gated, "bias": bias, "residual": residual, "train": train}


def listed():
    return [
        # the gate and up products of one generated token: reads the weights and little else
        _linear("linear_token_bf16", "bf16", 1, 11008, 4096, "silu", gated=True),
        # a handful of rows against a small odd-sized fp32 layer: latency
        _linear("linear_rows_f32", "f32", 13, 1021, 777, "relu", bias=True, residual=True),
        # a batch of 64 against a square weight, added to its residual
        _linear("linear_batch_bf16", "bf16", 64, 4096, 4096, "none", bias=True, residual=True),
        # an MLP's up-projection in training, pre-activations kept
        _linear("linear_mlp_bf16", "bf16", 4096, 11008, 4096, "gelu", bias=True, train=True),
        # odd extents everywhere: no row but the first begins on a 16-byte boundary
        _linear("linear_ragged_bf16", "bf16", 1999, 2623, 3457, "gelu", bias=True, residual=True),
        # the gradients of a square layer over 4096 tokens
        _linear_backward("linear_backward_bf16", "bf16", 4096, 4096, 4096, "gelu", bias=True),
        # the gradients of a gated odd-sized fp32 layer
        _linear_backward("linear_backward_f32", "f32", 999, 515, 1021, "silu", gated=True, bias=True),
        # the routing of a few generated tokens: latency
        _route("route_tokens_f32", "f32", 4, 64, 6, "softmax"),
        # the routing of a training batch: groups, a balancing bias, padded rows, and its gradient
        _route("route_train_bf16", "bf16", 16384, 256, 8, "sigmoid", groups=8, keep=4, bias=True,
               scale=2.5, train=True, shut=0.02),
        # one generated token through 6 of 64 experts
        _experts("experts_token_bf16", "experts", "bf16", 1, 64, 6, 2048, 1024, "silu", True,
                 residual=True),
        # a prompt through 2 of 8 wide experts
        _experts("experts_prompt_bf16", "experts", "bf16", 4096, 8, 2, 2048, 4096, "silu", True,
                 residual=True),
        # a training batch through 4 of 32 experts: all gradients
        _experts("experts_backward_bf16", "experts_backward", "bf16", 4096, 32, 4, 1024, 1024,
                 "silu", True, bias=True),
    ]


def _size(rng, lo, hi):
    """An extent in [lo, hi], spread over its logarithm: a third powers of two, a third multiples
    of 8, a third any number."""
    v = 2.0 ** rng.uniform(math.log2(lo), math.log2(hi))
    kind = rng.randrange(3)
    n = 2 ** round(math.log2(v)) if kind == 0 else 8 * round(v / 8) if kind == 1 else round(v)
    n = min(hi, max(lo, n))
    return n + 1 if n == 3072 else n


def _cost(case):
    w = work(case)
    return w["bytes"] / PRICE["bytes"] + w["flops"] / PRICE[case["dtype"]]


def _drawn(rng):
    op = rng.choice(("linear", "linear", "linear_backward", "route", "experts", "experts_backward"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    act = rng.choice(("none", "relu", "gelu", "silu"))
    gated, bias, residual, train = (rng.random() < 0.5 for _ in range(4))
    if op == "route":
        groups = rng.choice((1, 1, 2, 4, 8))
        E = groups * _size(rng, 2, 512 // groups)
        keep = rng.randint(1, groups)
        k = rng.randint(1, min(16, keep * (E // groups)))
        return _route("", dtype, _size(rng, 1, 16384), E, k, rng.choice(("softmax", "sigmoid")),
                      groups, keep, bias, rng.random() < 0.5, rng.choice((1.0, 2.5)), train,
                      rng.choice((0.0, 0.02)))
    if op.startswith("experts"):
        E = _size(rng, 2, 64)
        c = _experts("", op, dtype, _size(rng, 1, 4096), E, rng.randint(1, min(8, E)),
                     _size(rng, 64, 2048), _size(rng, 64, 4096), act, gated, bias)
        return {**c, "residual": residual, "train": train} if op == "experts" else c
    M, N, K = _size(rng, 1, 4096), _size(rng, 64, 11008), _size(rng, 64, 4096)
    if op == "linear":
        return _linear("", dtype, M, N, K, act, gated, bias, residual, train)
    return _linear_backward("", dtype, M, N, K, act, gated, bias)


def draw(rng):
    """Another case of the listed ranges (no name) that costs no more than the largest listed one,
    in fp32 no more than a quarter of it."""
    most = max(_cost(c) for c in listed())
    while True:
        c = _drawn(rng)
        if _cost(c) <= (most if c["dtype"] == "bf16" else most / 4):
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


def _lists(experts, E):
    """offsets [E+1], order [T·k] and place [T·k] of a table of experts (-1: none): the entries
    sorted by expert, each entry's place in that order."""
    flat = experts.reshape(-1).long()
    sorted_, order = torch.sort(torch.where(flat < 0, E, flat), stable=True)
    offsets = torch.searchsorted(sorted_, torch.arange(E + 1, device=flat.device))
    place = torch.empty_like(order)
    place[order] = torch.arange(order.numel(), device=flat.device)
    used = sorted_ < E
    return (offsets.int(), torch.where(used, order, -1).int(),
            torch.where(flat < 0, -1, place).int())


def prepare(case, seed):
    normal = _draws(seed)
    op, dt = case["op"], case["dtype"]
    s = {"case": case}
    if op.startswith("linear"):
        M, N, K = case["M"], case["N"], case["K"]
        wide = N * (2 if case["gated"] else 1)
        s["X"], s["W"] = normal(dt, M, K), normal(dt, K, wide, std=K ** -0.5)
        if op == "linear":
            s["bias"] = normal(dt, wide, std=0.1) if case["bias"] else None
            s["residual"] = normal(dt, M, N) if case["residual"] else None
        else:
            s["P"], s["dY"] = normal(dt, M, wide), normal(dt, M, N)
        return s
    T, E, k = case["T"], case["E"], case["k"]
    # experts are not equally liked: a spread of favour over them
    logits = (normal("f32", T, E, std=1.5) + normal("f32", E, std=0.5)).to(TYPES[dt])
    if op == "route":
        if case["shut"]:   # padded rows go to no expert
            logits[normal("f32", T) > 2.05] = -math.inf
        s["logits"] = logits
        s["bias"] = normal("f32", E, std=0.1) if case["bias"] else None
        s["dweights"] = normal("f32", T, k) if case["train"] else None
        return s
    D, H = case["D"], case["H"]
    wide = H * (2 if case["gated"] else 1)
    top, experts = torch.topk(logits.float(), k, dim=1)
    s["experts"], s["weights"] = experts.int().contiguous(), torch.softmax(top, dim=1)
    s["offsets"], s["order"], s["place"] = _lists(experts, E)
    s["X"] = normal(dt, T, D)
    s["W1"], s["W2"] = normal(dt, E, D, wide, std=D ** -0.5), normal(dt, E, H, D, std=H ** -0.5)
    s["b1"] = normal(dt, E, wide, std=0.1) if case["bias"] else None
    s["b2"] = normal(dt, E, D, std=0.1) if case["bias"] else None
    if op == "experts":
        s["residual"] = normal(dt, T, D) if case["residual"] else None
    else:   # the pre-activations that the forward pass left, in the order of the experts' rows
        s["P"], s["dY"] = normal(dt, T * k, wide), normal(dt, T, D)
    return s


# --------------------------------------------------------------------------------------------------
# the plain forms, in 32 bits
# --------------------------------------------------------------------------------------------------

def _f(t):
    return None if t is None else t.float()


def _act(x, act):
    if act == "relu":
        return torch.where(x > 0, x, 0.0)
    if act == "gelu":
        return 0.5 * x * (1 + torch.erf(x * 0.5 ** 0.5))
    if act == "silu":
        return x / (1 + torch.exp(-x))
    return x


def _slope(x, act):
    if act == "relu":
        return (x > 0).to(x.dtype)
    if act == "gelu":
        return (0.5 * (1 + torch.erf(x * 0.5 ** 0.5))
                + x * torch.exp(-0.5 * x * x) * (2 * math.pi) ** -0.5)
    if act == "silu":
        g = 1 / (1 + torch.exp(-x))
        return g * (1 + x * (1 - g))
    return torch.ones_like(x)


def _activate(P, act, gated):
    if not gated:
        return _act(P, act)
    n = P.shape[-1] // 2
    return _act(P[..., :n], act) * P[..., n:]


def _activate_backward(dH, P, act, gated):
    if not gated:
        return dH * _slope(P, act)
    n = P.shape[-1] // 2
    gate, up = P[..., :n], P[..., n:]
    return torch.cat((dH * up * _slope(gate, act), dH * _act(gate, act)), dim=-1)


def _plain_linear(s, c):
    dt = TYPES[c["dtype"]]
    P = s["X"].float() @ s["W"].float()
    if s["bias"] is not None:
        P = P + s["bias"].float()
    Y = _activate(P, c["act"], c["gated"])
    if s["residual"] is not None:
        Y = Y + s["residual"].float()
    return {"Y": Y.to(dt), "P": P.to(dt) if c["train"] else None}


def _plain_linear_backward(s, c):
    dt = TYPES[c["dtype"]]
    dP = _activate_backward(s["dY"].float(), s["P"].float(), c["act"], c["gated"])
    return {"dX": (dP @ s["W"].float().T).to(dt), "dW": (s["X"].float().T @ dP).to(dt),
            "db": dP.sum(0) if c["bias"] else None}


def _choose(key, c):
    """The k largest keys of every row, the lowest index first among equals; -1 for a key of -inf."""
    T, E = key.shape
    if c["groups"] > 1:
        per = torch.sort(key.view(T, c["groups"], -1), dim=2, descending=True).values
        best = per[:, :, 0] + per[:, :, 1] if per.shape[2] > 1 else per[:, :, 0]
        kept = torch.sort(best, dim=1, descending=True, stable=True).indices[:, :c["keep"]]
        mask = torch.zeros_like(best, dtype=torch.bool).scatter_(1, kept, True)
        key = torch.where(mask.repeat_interleave(E // c["groups"], dim=1), key, -math.inf)
    top, index = torch.sort(key, dim=1, descending=True, stable=True)
    return torch.where(top[:, :c["k"]] > -math.inf, index[:, :c["k"]], -1)


def _plain_route(s, c):
    logits = s["logits"].float()
    E, k = c["E"], c["k"]
    experts = _choose(logits if s["bias"] is None else logits + s["bias"], c)
    live, at = experts >= 0, experts.clamp(min=0)
    if c["score"] == "softmax":
        top = logits.amax(dim=1, keepdim=True)
        e = torch.exp(logits - torch.where(top > -math.inf, top, 0.0))
        score = e / e.sum(dim=1, keepdim=True).clamp(min=1e-30)
    else:
        score = 1 / (1 + torch.exp(-logits))
    chosen = torch.where(live, score.gather(1, at), 0.0)
    total = chosen.sum(dim=1, keepdim=True).clamp(min=1e-30) if c["renormalise"] else 1.0
    part = chosen / total
    offsets, order, place = _lists(experts, E)
    out = {"weights": c["scale"] * part, "experts": experts.int(), "offsets": offsets,
           "order": order, "place": place.view(-1, k)}
    if s["dweights"] is not None:
        dw = torch.where(live, c["scale"] * s["dweights"], 0.0)
        mean = (dw * part).sum(dim=1, keepdim=True)
        if c["score"] == "sigmoid":
            d = part * (1 - chosen) * (dw - mean if c["renormalise"] else dw)
            d = torch.zeros_like(logits).scatter_add_(1, at, torch.where(live, d, 0.0))
        else:
            d = torch.zeros_like(logits).scatter_add_(1, at, part * (dw - mean) if c["renormalise"]
                                                      else part * dw)
            if not c["renormalise"]:
                d = d - score * mean
        out["dlogits"] = d.to(s["logits"].dtype)
    return out


def _table(s, c):
    """Rows of the experts' inputs in a table [E, most, ...] (most: the fullest expert's rows), as
    the table's shape, each sorted row's cell in it, and its token and slot."""
    E, R = c["E"], c["T"] * c["k"]
    counts = s["offsets"][1:] - s["offsets"][:-1]
    most = int(counts.max())
    order = s["order"].long()
    expert = s["experts"].reshape(-1)[order].long()
    cell = expert * most + torch.arange(R, device=order.device) - s["offsets"][expert].long()
    return most, cell, order // c["k"], expert


def _fill(rows, cell, E, most):
    t = torch.zeros(E * most, rows.shape[1], device=rows.device)
    t[cell] = rows
    return t.view(E, most, -1)


def _plain_experts(s, c):
    dt = TYPES[c["dtype"]]
    E, T, k = c["E"], c["T"], c["k"]
    most, cell, token, expert = _table(s, c)
    X = s["X"].float()[token]
    if T * k <= E:   # few rows: each with the weights of its expert
        P = torch.bmm(X.unsqueeze(1), s["W1"][expert].float()).squeeze(1)
    else:
        P = torch.bmm(_fill(X, cell, E, most), s["W1"].float()).flatten(0, 1)[cell]
    if s["b1"] is not None:
        P = P + s["b1"].float()[expert]
    H = _activate(P, c["act"], c["gated"])
    if T * k <= E:
        O = torch.bmm(H.unsqueeze(1), s["W2"][expert].float()).squeeze(1)
    else:
        O = torch.bmm(_fill(H, cell, E, most), s["W2"].float()).flatten(0, 1)[cell]
    if s["b2"] is not None:
        O = O + s["b2"].float()[expert]
    Y = (O[s["place"].long()].view(T, k, -1) * s["weights"].unsqueeze(2)).sum(1)
    if s["residual"] is not None:
        Y = Y + s["residual"].float()
    return {"Y": Y.to(dt), "P": P.to(dt) if c["train"] else None}


def _plain_experts_backward(s, c):
    dt = TYPES[c["dtype"]]
    E, T, k = c["E"], c["T"], c["k"]
    most, cell, token, expert = _table(s, c)
    w = s["weights"].reshape(-1)[s["order"].long()].unsqueeze(1)
    P, W1, W2 = s["P"].float(), s["W1"].float(), s["W2"].float()
    dY, X = s["dY"].float()[token], s["X"].float()[token]
    H = _activate(P, c["act"], c["gated"])
    dO = _fill(w * dY, cell, E, most)
    dH = torch.bmm(_fill(dY, cell, E, most), W2.transpose(1, 2).contiguous()).flatten(0, 1)[cell]
    dw = (dH * H).sum(1)
    dP = _fill(_activate_backward(w * dH, P, c["act"], c["gated"]), cell, E, most)
    dX = torch.bmm(dP, W1.transpose(1, 2).contiguous()).flatten(0, 1)[cell]
    dX = dX[s["place"].long()].view(T, k, -1).sum(1)
    dW2 = torch.bmm(_fill(H, cell, E, most).transpose(1, 2).contiguous(), dO)
    dW1 = torch.bmm(_fill(X, cell, E, most).transpose(1, 2).contiguous(), dP)
    if c["bias"]:
        dw = dw + (dY * s["b2"].float()[expert]).sum(1)
    return {"dX": dX.to(dt), "dW1": dW1.to(dt), "dW2": dW2.to(dt),
            "db1": dP.sum(1) if c["bias"] else None, "db2": dO.sum(1) if c["bias"] else None,
            "dweights": dw[s["place"].long()].view(T, k)}


# --------------------------------------------------------------------------------------------------
# the framework's calls
# --------------------------------------------------------------------------------------------------

def _own(s, c):
    from paper_1909_10616_amd import layers
    op = c["op"]
    if op == "linear":
        X, W = s["X"], s["W"]
        P = torch.empty(X.shape[0], W.shape[1], dtype=X.dtype, device=X.device) if c["train"] else None
        Y = layers.gt_linear(X, W, bias=s["bias"], residual=s["residual"], act=c["act"],
                             gated=c["gated"], P=P)
        return {"Y": Y, "P": P}
    if op == "linear_backward":
        dX, dW, db = layers.gt_linear_backward(s["dY"], s["X"], s["W"], P=s["P"], act=c["act"],
                                               gated=c["gated"], bias=c["bias"])
        return {"dX": dX, "dW": dW, "db": db}
    if op == "route":
        how = {"score": c["score"], "renormalise": c["renormalise"], "scale": c["scale"]}
        r = layers.gt_route(s["logits"], c["k"], bias=s["bias"], groups=c["groups"], keep=c["keep"],
                            **how)
        out = r._asdict()
        if s["dweights"] is not None:
            out["dlogits"] = layers.gt_route_backward(s["dweights"], s["logits"], r.experts, **how)
        return out
    r = layers.Route(s["weights"], s["experts"], s["offsets"], s["order"],
                     s["place"].view(c["T"], c["k"]))
    if op == "experts":
        P = None
        if c["train"]:
            P = torch.empty(c["T"] * c["k"], s["W1"].shape[2], dtype=s["X"].dtype,
                            device=s["X"].device)
        Y = layers.gt_experts(s["X"], r, s["W1"], s["W2"], b1=s["b1"], b2=s["b2"],
                              residual=s["residual"], act=c["act"], gated=c["gated"], P=P)
        return {"Y": Y, "P": P}
    g = layers.gt_experts_backward(s["dY"], s["X"], r, s["W1"], s["W2"], s["P"], b2=s["b2"],
                                   act=c["act"], gated=c["gated"], bias=c["bias"])
    return g._asdict()


PLAIN = {"linear": _plain_linear, "linear_backward": _plain_linear_backward, "route": _plain_route,
         "experts": _plain_experts, "experts_backward": _plain_experts_backward}


def run(state):
    case = state["case"]
    return _own(state, case) if own else PLAIN[case["op"]](state, case)


# --------------------------------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------------------------------

def work(case):
    op, size = case["op"], SIZE[case["dtype"]]
    if op.startswith("linear"):
        M, N, K = case["M"], case["N"], case["K"]
        wide = N * (2 if case["gated"] else 1)
        if op == "linear":
            values = M * K + K * wide + M * N * (2 if case["residual"] else 1)
            values += (wide if case["bias"] else 0) + (M * wide if case["train"] else 0)
            return {"bytes": values * size, "flops": 2 * M * wide * K}
        # X, W, P (where the activation has a slope) and dY in, dX and dW out, db in 32 bits
        saved = M * wide if case["gated"] or case["act"] != "none" else 0
        values = 2 * (M * K + K * wide) + saved + M * N
        return {"bytes": values * size + (wide * 4 if case["bias"] else 0),
                "flops": 4 * M * wide * K}
    T, E, k = case["T"], case["E"], case["k"]
    if op == "route":
        nbytes = T * E * size + 16 * T * k + 4 * (E + 1) + (4 * E if case["bias"] else 0)
        if case["train"]:   # the same logits and experts read, dweights read, dlogits written
            nbytes += T * E * size * 2 + 8 * T * k
        return {"bytes": nbytes, "flops": T * E * (8 if case["train"] else 4)}
    D, H, R = case["D"], case["H"], T * k
    wide = H * (2 if case["gated"] else 1)
    used = E * (1 - (1 - k / E) ** T)   # experts that get a row, were all alike
    weights = used * (D * wide + H * D)
    lists = 16 * R + 4 * (E + 1)
    products = 2 * R * (D * wide + H * D)
    if op == "experts":
        values = T * D * (3 if case["residual"] else 2) + weights + (R * wide if case["train"] else 0)
        values += used * (wide + D) if case["bias"] else 0
        return {"bytes": values * size + lists, "flops": products}
    values = 3 * T * D + R * wide + weights + E * (D * wide + H * D)
    if case["bias"]:
        lists += E * (wide + D) * 4 + E * D * size
    return {"bytes": values * size + lists + 4 * R, "flops": 2 * products}


# --------------------------------------------------------------------------------------------------
# the definitions, in 64 bits
# --------------------------------------------------------------------------------------------------

def _value_and_slope(x, act):
    """An activation and its derivative."""
    if act == "none":
        return x, torch.ones_like(x)
    if act == "relu":
        return x.clamp(min=0), torch.heaviside(x, torch.zeros_like(x))
    if act == "silu":
        g = torch.sigmoid(x)
        return x * g, g + x * g * (1 - g)
    cdf = torch.special.ndtr(x)
    return x * cdf, cdf + x * torch.exp(-x ** 2 / 2) / math.sqrt(2 * math.pi)


def _hidden(P, case):
    """The activated rows and the factors that turn dH into dP: one, or the gate's and the up's."""
    if not case["gated"]:
        h, d = _value_and_slope(P, case["act"])
        return h, (d,)
    gate, up = P.chunk(2, dim=1)
    h, d = _value_and_slope(gate, case["act"])
    return h * up, (up * d, h)


def exact(case, seed):
    s = {n: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v
         for n, v in prepare(case, seed).items()}
    op = case["op"]
    if op == "linear":
        P = torch.mm(s["X"], s["W"])
        P += 0 if s["bias"] is None else s["bias"]
        Y, _ = _hidden(P, case)
        return {"Y": Y if s["residual"] is None else Y + s["residual"],
                "P": P if case["train"] else None}
    if op == "linear_backward":
        dP = torch.cat([f * s["dY"] for f in _hidden(s["P"], case)[1]], dim=1)
        return {"dX": torch.mm(dP, s["W"].t()), "dW": torch.mm(s["X"].t(), dP),
                "db": dP.sum(dim=0) if case["bias"] else None}
    if op == "route":
        return _exact_route(case, s)
    return _exact_experts(case, s)


def _exact_route(case, s):
    logits, E, k = s["logits"], case["E"], case["k"]
    # the key is the float32 sum of logit and bias, the score of a group the float32 sum of two keys
    key = logits.float() if s["bias"] is None else (logits + s["bias"]).float()
    T = key.shape[0]
    if case["groups"] > 1:
        best = torch.topk(key.view(T, case["groups"], -1).double(), min(2, E // case["groups"]),
                          dim=2).values.sum(dim=2).float()
        beaten_by = (best.unsqueeze(1) > best.unsqueeze(2)).sum(dim=2)
        tied = best.unsqueeze(1) == best.unsqueeze(2)
        beaten_by += torch.tril(tied.int(), diagonal=-1).sum(dim=2)   # equals of a lower index
        open_ = (beaten_by < case["keep"]).repeat_interleave(E // case["groups"], dim=1)
        key = key.masked_fill(~open_, -math.inf)
    # k times the largest key left; argmax takes the first of equals on the CPU
    key, experts = key.cpu().clone(), []
    for _ in range(k):
        best, at = key.max(dim=1)
        first = (key == best.unsqueeze(1)).int().argmax(dim=1)
        experts.append(torch.where(best > -math.inf, first, -1))
        key.scatter_(1, first.unsqueeze(1), -math.inf)
    experts = torch.stack(experts, dim=1).to(logits.device)
    live = experts >= 0
    hot = torch.zeros(T, k, E, device=logits.device, dtype=torch.bool)
    hot.scatter_(2, experts.clamp(min=0).unsqueeze(2), live.unsqueeze(2))
    if case["score"] == "softmax":
        score = torch.softmax(logits, dim=1).nan_to_num(0.0)
        slope = None
    else:
        score = torch.sigmoid(logits)
        slope = score * (1 - score)
    chosen = (hot * score.unsqueeze(1)).sum(dim=2)
    total = chosen.sum(dim=1, keepdim=True)
    total = torch.where(total > 0, total, 1.0) if case["renormalise"] else torch.ones_like(total)
    weights = case["scale"] * chosen / total
    flat = experts.flatten().tolist()
    rows = sorted((e, i) for i, e in enumerate(flat) if e >= 0)
    counts = [0] * (E + 1)
    place = [-1] * len(flat)
    for n, (e, i) in enumerate(rows):
        counts[e + 1] += 1
        place[i] = n
    order = [i for _, i in rows] + [-1] * (len(flat) - len(rows))
    whole = lambda v: torch.tensor(v, dtype=torch.int32, device=logits.device)  # noqa: E731
    out = {"weights": weights, "experts": experts.int(), "offsets": whole(counts).cumsum(0).int(),
           "order": whole(order), "place": whole(place).view(T, k)}
    if s["dweights"] is not None:
        # through the quotient to the scores, then through the scores to the logits
        dw = s["dweights"] * case["scale"] / total
        if case["renormalise"]:
            dw = dw - (dw * chosen).sum(dim=1, keepdim=True) / total
        d = (hot * dw.unsqueeze(2)).sum(dim=1)
        out["dlogits"] = d * slope if slope is not None else \
            score * (d - (d * score).sum(dim=1, keepdim=True))
    return out


def _exact_experts(case, s):
    T, E, k = case["T"], case["E"], case["k"]
    bounds, order = s["offsets"].tolist(), s["order"].long()
    out = {n: torch.zeros(T * k, s[n].shape[-1], device=order.device, dtype=torch.float64)
           for n in ("W1", "X")}
    P, O = out["W1"], out["X"]
    w = s["weights"].flatten()[order]
    forward = case["op"] == "experts"
    g = None if forward else {n: torch.zeros_like(s[n]) for n in ("X", "W1", "W2")}
    db1, db2 = ([], [])
    dw = torch.zeros(T * k, device=order.device, dtype=torch.float64)
    for e in range(E):
        mine = slice(bounds[e], bounds[e + 1])
        token = order[mine] // k
        if forward:
            P[mine] = s["X"][token] @ s["W1"][e] + (0 if s["b1"] is None else s["b1"][e])
            O[mine] = _hidden(P[mine], case)[0] @ s["W2"][e] + (0 if s["b2"] is None else s["b2"][e])
            continue
        h, factors = _hidden(s["P"][mine], case)
        dO = s["dY"][token] * w[mine, None]
        dH = dO @ s["W2"][e].t()
        dP = torch.cat([f * dH for f in factors], dim=1)
        # the weight's gradient is dY·(the expert's output)
        dw[order[mine]] = (s["dY"][token] * (h @ s["W2"][e] + (s["b2"][e] if case["bias"] else 0))
                           ).sum(dim=1)
        g["W2"][e], g["W1"][e] = h.t() @ dO, s["X"][token].t() @ dP
        g["X"].index_add_(0, token, dP @ s["W1"][e].t())
        db1.append(dP.sum(dim=0))
        db2.append(dO.sum(dim=0))
    if forward:
        Y = torch.zeros_like(s["X"]) if s["residual"] is None else s["residual"].clone()
        Y.index_add_(0, order // k, O * w[:, None])
        return {"Y": Y, "P": P if case["train"] else None}
    return {"dX": g["X"], "dW1": g["W1"], "dW2": g["W2"],
            "db1": torch.stack(db1) if case["bias"] else None,
            "db2": torch.stack(db2) if case["bias"] else None, "dweights": dw.view(T, k)}
