"""The layer operators' definitions in 64 bits on the CPU, for the tests, with
bounds on what 32-bit sums and the stated roundings may change.

A sum of n products formed in any order in fp32 is off by at most (n + 2)·2^-24
times the sum of the products' magnitudes. A value stored in type T is off by
u(T) of itself (2^-8 for bf16, half an ulp doubled; 2^-23 for fp32).
Activations have slopes of at most 1.13 and are evaluated to 16 ulp (the
exponential, the error function and a 1-ulp reciprocal)."""
import math

import torch

EPS = 2.0 ** -24
SLOPE = 1.13


def u(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -23


def d(t):
    return None if t is None else t.detach().cpu().double()


def act(x, name):
    if name == "relu":
        return torch.where(x < 0, 0.0, x)
    if name == "gelu":
        return 0.5 * x * (1 + torch.erf(x / math.sqrt(2)))
    if name == "silu":
        return x * torch.sigmoid(x)
    return x


def slope(x, name):
    if name == "relu":
        return (x > 0).double()
    if name == "gelu":
        return 0.5 * (1 + torch.erf(x / math.sqrt(2))) + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = torch.sigmoid(x)
        return s * (1 + x * (1 - s))
    return torch.ones_like(x)


def product(A, B, dA=None, dB=None):
    """A·B and its bound, given the operands' own errors."""
    n = A.shape[-1]
    err = (n + 2) * EPS * (A.abs() @ B.abs())
    if dA is not None:
        err = err + dA @ B.abs()
    if dB is not None:
        err = err + A.abs() @ dB
    return A @ B, err


def activate(P, dP, name, gated):
    """act(P) (gated: act(gate)·up) and its bound."""
    if not gated:
        v = act(P, name)
        return v, (SLOPE if name != "none" else 1) * dP + 16 * EPS * (v.abs() + (P.abs() if name != "none" else 0))
    g, up = P.chunk(2, dim=-1)
    dg, du = dP.chunk(2, dim=-1)
    v, dv = activate(g, dg, name, False)
    return v * up, dv * (up.abs() + du) + v.abs() * du + EPS * (v * up).abs()


def stored(v, err, dtype):
    return v, err + u(dtype) * (v.abs() + err) + (2.0 ** -133 if dtype == torch.bfloat16 else 2.0 ** -126)


def linear(X, W, bias=None, residual=None, name="none", gated=False, dtype=None, out=None):
    dtype = dtype or X.dtype
    P, dP = product(d(X), d(W))
    if bias is not None:
        P = P + d(bias)
        dP = dP + 2 * EPS * P.abs()
    Y, dY = activate(P, dP, name, gated)
    if residual is not None:
        Y = Y + d(residual)
        dY = dY + 2 * EPS * Y.abs()
    return stored(Y, dY, out or dtype), stored(P, dP, dtype)


def act_grad(dH, err, P, name, gated):
    """dP and its bound from dH and its bound; P exact."""
    if not gated:
        s = slope(P, name)
        return dH * s, err * s.abs() + 32 * EPS * dH.abs() * (1 + P.abs())
    g, up = P.chunk(2, dim=-1)
    s, v = slope(g, name), act(g, name)
    dg = dH * up * s
    du = dH * v
    return torch.cat((dg, du), -1), torch.cat(
        (err * (up * s).abs() + 32 * EPS * (dH * up).abs() * (1 + g.abs()),
         err * v.abs() + 32 * EPS * dH.abs() * (v.abs() + g.abs())), -1)


def linear_backward(dY, X, W, P, name, gated, dtype, dw=None):
    dY, X, W = d(dY), d(X), d(W)
    dP, err = (dY, torch.zeros_like(dY)) if name == "none" and not gated else \
        act_grad(dY, torch.zeros_like(dY), d(P), name, gated)
    db = (dP.sum(0), err.sum(0) + (dP.shape[0] + 2) * EPS * dP.abs().sum(0) + 2.0 ** -126)
    rounded = torch.zeros_like(err) if name == "none" and not gated else stored(dP, err, dtype)[1]
    return (stored(*product(dP, W.T, dA=rounded), dtype),
            stored(*product(X.T, dP, dB=rounded), dw or dtype), db)


def choose(logits, k, bias, groups, keep):
    """[T][k] experts by the definition, one token at a time."""
    x = logits.detach().cpu().float()
    key = x if bias is None else x + bias.cpu()
    key = torch.where(torch.isnan(key) | torch.isnan(x), -math.inf, key)
    T, E = key.shape
    out = []
    for t in range(T):
        row = key[t]
        allowed = list(range(E))
        if groups > 1:
            size = E // groups
            scores = []
            for g in range(groups):
                top = sorted(row[g * size:(g + 1) * size].tolist(), reverse=True)[:2]
                s = torch.tensor(top, dtype=torch.float32).sum().item()
                scores.append(-math.inf if math.isnan(s) else s)
            kept = sorted(range(groups), key=lambda g: (-scores[g], g))[:keep]
            allowed = [e for e in allowed if e // size in kept]
        best = sorted((e for e in allowed if row[e] > -math.inf), key=lambda e: (-row[e].item(), e))[:k]
        out.append(best + [-1] * (k - len(best)))
    return torch.tensor(out, dtype=torch.int64).view(T, k)


def shares(logits, experts, score, renormalise):
    """Each chosen logit's share (the weight over scale), and the scores."""
    x = d(logits)
    x = torch.where(torch.isnan(x), -math.inf, x)
    live, at = experts >= 0, experts.clamp(min=0)
    c = x.gather(1, at) if x.shape[0] else x.new_zeros(experts.shape)
    top = x.amax(1, keepdim=True) if x.shape[0] else x.new_zeros(0, 1)
    e = torch.where(x == top, 1.0, torch.exp(x - top))
    e = torch.where(x > -math.inf, e, 0.0)
    soft = e / e.sum(1, keepdim=True).clamp(min=1e-300)
    if score == "softmax" and renormalise:
        m = torch.where(live, c, -math.inf).amax(1, keepdim=True)
        q = torch.where(live, torch.where(c == m, 1.0, torch.exp(c - m)), 0.0)
        return q / q.sum(1, keepdim=True).clamp(min=1e-300), soft
    if score == "softmax":
        return torch.where(live, soft.gather(1, at), 0.0), soft
    sig = torch.sigmoid(c)
    if renormalise:
        ls = torch.where(live, torch.nn.functional.logsigmoid(c), -math.inf)
        m = ls.amax(1, keepdim=True)
        q = torch.where(live, torch.exp(ls - torch.where(m > -math.inf, m, 0.0)), 0.0)
        return q / q.sum(1, keepdim=True).clamp(min=1e-300), sig
    return torch.where(live, sig, 0.0), sig


def lists(experts, E):
    flat = experts.flatten().tolist()
    rows = sorted((e, i) for i, e in enumerate(flat) if e >= 0)
    offsets = [0] * (E + 1)
    place = [-1] * len(flat)
    for n, (e, i) in enumerate(rows):
        offsets[e + 1] += 1
        place[i] = n
    for e in range(E):
        offsets[e + 1] += offsets[e]
    order = [i for _, i in rows] + [-1] * (len(flat) - len(rows))
    return (torch.tensor(offsets, dtype=torch.int32), torch.tensor(order, dtype=torch.int32),
            torch.tensor(place, dtype=torch.int32).view(experts.shape))


def route_backward(logits, experts, dweights, score, renormalise, scale):
    part, sc = shares(logits, experts, score, renormalise)
    live = experts >= 0
    g = torch.where(live, scale * d(dweights), 0.0)
    mean = (part * g).sum(1, keepdim=True)
    x = d(logits)
    out, size = torch.zeros_like(x), torch.zeros_like(x)
    if score == "sigmoid":
        v = part * (1 - sc) * (g - mean if renormalise else g)
    else:
        v = part * (g - mean if renormalise else g)
    out.scatter_add_(1, experts.clamp(min=0), torch.where(live, v, 0.0))
    size.scatter_add_(1, experts.clamp(min=0), torch.where(live, part * (g.abs() + (part * g.abs()).sum(1, keepdim=True)), 0.0))
    if score == "softmax" and not renormalise:
        out -= sc * mean
        size += sc * (part * g.abs()).sum(1, keepdim=True)
    return out, size


def experts(X, W1, W2, weights, chosen, order, b1, b2, residual, name, gated, dtype):
    """Y and P (in the order of the experts' rows) with their bounds."""
    Xd, w = d(X), d(weights)
    T, k = chosen.shape
    n = int((order >= 0).sum())
    wide, D = W1.shape[2], W2.shape[2]
    P = torch.zeros(n, wide, dtype=torch.float64)
    dP = torch.zeros_like(P)
    Y = torch.zeros(T, D, dtype=torch.float64) if residual is None else d(residual).clone()
    err = torch.zeros(T, D, dtype=torch.float64)
    size = Y.abs()
    for e in range(W1.shape[0]):
        rows = [p for p in range(n) if int(chosen.flatten()[order[p]]) == e]
        if not rows:
            continue
        ent = order[rows].long()
        tok = ent // k
        p, dp = product(Xd[tok], d(W1[e]))
        if b1 is not None:
            p = p + d(b1[e])
            dp = dp + 2 * EPS * p.abs()
        P[rows], dP[rows] = p, dp
        H, dH = stored(*activate(p, dp, name, gated), dtype)
        O, dO = product(H, d(W2[e]), dA=dH)
        if b2 is not None:
            O = O + d(b2[e])
            dO = dO + 2 * EPS * O.abs()
        ww = w.flatten()[ent][:, None]
        Y.index_add_(0, tok, O * ww)
        err.index_add_(0, tok, dO * ww.abs())
        size.index_add_(0, tok, (O * ww).abs())
    err += (k + 3) * EPS * size
    return stored(Y, err, dtype), stored(P, dP, dtype)


def experts_backward(dY, X, W1, W2, P, weights, chosen, order, b2, name, gated, dtype):
    """{name: (value, bound)} of all gradients."""
    dYd, Xd, Pd, w = d(dY), d(X), d(P), d(weights)
    T, k = chosen.shape
    E, D, wide = W1.shape
    H_ = W2.shape[1]
    z = lambda *s: torch.zeros(*s, dtype=torch.float64)  # noqa: E731
    out = {"dX": [z(T, D), z(T, D)], "dW1": [z(E, D, wide), z(E, D, wide)],
           "dW2": [z(E, H_, D), z(E, H_, D)], "db1": [z(E, wide), z(E, wide)],
           "db2": [z(E, D), z(E, D)], "dweights": [z(T * k), z(T * k)]}
    n = int((order >= 0).sum())
    for e in range(E):
        rows = [p for p in range(n) if int(chosen.flatten()[order[p]]) == e]
        if not rows:
            continue
        ent = order[rows].long()
        tok = ent // k
        ww = w.flatten()[ent][:, None]
        g = dYd[tok]
        dH, edH = product(g, d(W2[e]).T)
        H, eH = activate(Pd[rows], torch.zeros_like(Pd[rows]), name, gated)
        dP, edP = act_grad(dH * ww, edH * ww.abs() + EPS * (dH * ww).abs(), Pd[rows], name, gated)
        rP = stored(dP, edP, dtype)[1]
        out["db1"][0][e], out["db1"][1][e] = dP.sum(0), edP.sum(0) + (len(rows) + 2) * EPS * dP.abs().sum(0)
        out["db2"][0][e] = (g * ww).sum(0)
        out["db2"][1][e] = (len(rows) + 3) * EPS * (g * ww).abs().sum(0)
        Hw, eHw = stored(H * ww, eH * ww.abs() + EPS * (H * ww).abs(), dtype)
        out["dW2"][0][e], out["dW2"][1][e] = product(Hw.T, g, dA=eHw.T)
        out["dW1"][0][e], out["dW1"][1][e] = product(Xd[tok].T, dP, dB=rP)
        dx, ex = product(dP, d(W1[e]).T, dA=rP)
        out["dX"][0].index_add_(0, tok, dx)
        out["dX"][1].index_add_(0, tok, ex + (k + 2) * EPS * dx.abs())
        dw = (dH * H).sum(1)
        ew = (edH * H.abs() + dH.abs() * eH).sum(1) + (H_ + 2) * EPS * (dH * H).abs().sum(1)
        if b2 is not None:
            dw = dw + g @ d(b2[e])
            ew = ew + (D + 2) * EPS * (g.abs() @ d(b2[e]).abs()) + 2 * EPS * dw.abs()
        out["dweights"][0][ent], out["dweights"][1][ent] = dw, ew
    for name_ in ("dX", "dW1", "dW2"):
        out[name_] = list(stored(*out[name_], dtype))
    for name_ in ("db1", "db2", "dweights"):
        out[name_][1] = out[name_][1] + 2.0 ** -126 + 2.0 ** -23 * out[name_][0].abs()
    out["dweights"] = [v.view(T, k) for v in out["dweights"]]
    return out


def check(got, want, what):
    """Every value of got within its bound."""
    value, bound = want
    g = d(got)
    assert g.shape == value.shape, (what, g.shape, value.shape)
    bad = ~((g - value).abs() <= bound)
    if bool(bad.any()):
        at = tuple(int(i) for i in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} out of bounds, first {at}: "
                             f"{g[at].item()!r} for {value[at].item()!r} ± {bound[at].item():.3g}")
