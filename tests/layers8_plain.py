"""The norm, the quantising and the 8-bit layers in plain form on the CPU, for the tests, with
bounds on what 32-bit steps may change.

Codes and scales are whole steps of 32-bit arithmetic and have to be the same bits. The other
values are computed in 64 bits; E = 2^-24 is one rounding to fp32.

A sum of n terms in fp32, in any order, is off by at most (n - 1)·E times the terms' magnitudes
(first order; a second E a term covers the higher ones at these lengths); the norm's
sums over a row go by trees, whose longest chain CHAIN counts."""
import torch

import layers_plain as ref
from layers_plain import EPS as E
from layers_plain import d

FP8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
LARGEST = {torch.float8_e4m3fn: 448.0, torch.float8_e5m2: 57344.0}


def blocks(n):
    return -(-n // 128)


def widen(s, rows, cols, block):
    """A scale for each value."""
    s = s.repeat_interleave(128, dim=1)[:, :cols]
    return s.repeat_interleave(128, dim=0)[:rows] if block == "square" else s


def quantise(X, block, code, pow2=False):
    """Codes and scales of X (float32 or bfloat16): NaN left out of the maxima."""
    x = X.detach().cpu().float()
    M, N = x.shape
    b, m = blocks(N), blocks(M)
    size = torch.zeros(M if block == "row" else m * 128, b * 128)
    size[:M, :N] = torch.where(torch.isnan(x), 0.0, x.abs())
    most = size.view(-1, b, 128).amax(2) if block == "row" else size.view(m, 128, b, 128).amax((1, 3))
    s = (most / LARGEST[FP8[code]]).clamp(min=2.0 ** -126)
    if pow2:
        bits = s.view(torch.int32)
        s = ((bits + 0x7fffff) & 0x7f800000).view(torch.float32)
    s = torch.where(most == 0, 1.0, s)
    return (x * widen(1.0 / s, M, N, block)).to(FP8[code]), s


def same_codes(got, want):
    """Equal bits, but for the sign of NaN."""
    a, b = got.cpu().float(), want.float()
    return got.dtype == want.dtype and bool(((a == b) & (torch.signbit(a) == torch.signbit(b)) |
                                             (torch.isnan(a) & torch.isnan(b))).all())


# ---- norm

def chain(N):
    """Additions in a row's longest chain: 3 in an octet, up to 4 octets of a thread (or a long row's octets of
    1024 threads), 6 over a wavefront, up to 16 over the wavefronts; and the division."""
    octets = 4 if N <= 16384 else blocks(N) / 64 + 1
    return 3 + octets + 6 + 16 + 1


def stats(X, eps):
    x = d(X)
    mean = x.mean(1, keepdim=True)
    var = ((x - mean) ** 2).mean(1, keepdim=True)
    rstd = (var + eps) ** -0.5
    g = 2 * chain(x.shape[1]) * E
    dmean = g * x.abs().mean(1, keepdim=True)
    # of rstd, relative: half the variance's: its sum, its terms' three roundings, the mean's error squared
    # (the deviations sum to zero, so that it enters in second order); root, sum with eps, reciprocal
    away = (x - mean).abs() + dmean
    drstd = 0.5 * (g + 4 * E) + 0.5 * (dmean * rstd) ** 2 + dmean * rstd * rstd * 2 * E * away.mean(1, keepdim=True) + 4 * E
    return x, mean, rstd, dmean, drstd


def norm(X, w, b, eps, dtype):
    """(Y, its bound), (mean, bound), (rstd, bound); Y as stored in dtype, or before it (None)."""
    x, mean, rstd, dmean, drstd = stats(X, eps)
    w = d(w) if w is not None else torch.ones(x.shape[1], dtype=torch.float64)
    b = d(b) if b is not None else torch.zeros(x.shape[1], dtype=torch.float64)
    h = (x - mean) * rstd
    err = (w.abs() * rstd * (dmean + E * ((x - mean).abs() + dmean)) * (1 + drstd) + (w * h).abs() * (drstd + 3 * E)
           + E * ((w * h).abs() + b.abs()) * 2 + 2.0 ** -126)
    y = h * w + b
    out = (y, err) if dtype is None else ref.stored(y, err, dtype)
    return (out, (mean.squeeze(1), (dmean + E * mean.abs() + 2.0 ** -126).squeeze(1)),
            (rstd.squeeze(1), (drstd * rstd).squeeze(1)))


def norm_backward(dY, X, mean, rstd, w, R, dtype):
    """(dX, bound), (dw, bound), (db, bound) of these 32-bit statistics."""
    dY, x = d(dY), d(X)
    mean, rstd = d(mean).unsqueeze(1), d(rstd).unsqueeze(1)
    w = d(w) if w is not None else torch.ones(x.shape[1], dtype=torch.float64)
    M, N = x.shape
    g = 2 * chain(N) * E
    h = (x - mean) * rstd
    dh = 2 * E * h.abs()
    gr = dY * w
    m1, m2 = gr.mean(1, keepdim=True), (gr * h).mean(1, keepdim=True)
    e1 = (g + 3 * E) * gr.abs().mean(1, keepdim=True)
    e2 = (g + 6 * E) * (gr * h).abs().mean(1, keepdim=True)
    err = rstd * (E * gr.abs() + e1 + h.abs() * e2 + dh * m2.abs() + 4 * E * (gr.abs() + m1.abs() + (h * m2).abs()))
    dX = rstd * (gr - m1 - h * m2)
    if R is not None:
        dX = dX + d(R)
        err = err + 2 * E * (dX.abs() + d(R).abs())
    rows = 2 * (M + 32) * E
    dw = ((dY * h).sum(0), (rows + 4 * E) * (dY * h).abs().sum(0) + 2.0 ** -126)
    db = (dY.sum(0), rows * dY.abs().sum(0) + 2.0 ** -126)
    return ref.stored(dX, err + 2.0 ** -126, dtype), dw, db


# ---- linear of codes

def linear(X, sx, W, sw, xblock="row", wblock="square", bias=None, residual=None, act="none", gated=False,
           dtype=torch.bfloat16):
    """Y and its bound. Products of two codes are exact in fp32 (4 + 4 significant bits at most). Where Y is
    fp32, a block's sum of 128 is taken to be off by a whole last place, 2E, of the magnitudes at each of its
    additions. Where it is bf16, the instruction may drop what lies 13 bits below the largest of 8 products that
    it adds at once: each of the 8 is off by at most 2^-13 of it, their sum by 8·2^-13 = 2^-10 of their
    magnitudes. Then the scales' product, its product with the sum and one addition a block."""
    M, K = X.shape
    wide = W.shape[0]
    x, w = X.cpu().float().double(), W.cpu().float().double()
    xs, ws = widen(d(sx), M, K, xblock), widen(d(sw), wide, K, wblock)
    a, b = x * xs, w * ws
    P = a @ b.T
    dP = ((2.0 ** -10 if dtype == torch.bfloat16 else 0) + (2 * 128 + 2 * (blocks(K) + 12)) * E) * (a.abs() @ b.abs().T)
    if bias is not None:
        P = P + d(bias)
        dP = dP + 2 * E * P.abs()
    Y, dY = ref.activate(P, dP, act, gated)
    if residual is not None:
        Y = Y + d(residual)
        dY = dY + 2 * E * Y.abs()
    return ref.stored(Y, dY, dtype)
