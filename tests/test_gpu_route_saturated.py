"""The gradient of sigmoid scores that are almost 1, or almost 0: σ'(x) = σ(x)·σ(−x) to the last
bits, where 1 − σ(x) has none."""
import math

import pytest
import torch

import layers_plain as ref
from test_gpu_layers import BF16, F32, IDS, L  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("renormalise", [False, True])
# (T, E, k): a row of 16 lanes a token, and a wavefront a token
@pytest.mark.parametrize("case", [(60, 16, 4), (40, 128, 8), (33, 256, 16), (30, 300, 5), (20, 64, 20)], ids=str)
@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS.get)
def test_route_backward(L, dtype, case, renormalise):  # noqa: F811
    T, E, k = case
    gen = torch.Generator().manual_seed(E)
    # each token about a level of its own, from −60 to 60
    x = (torch.randn(T, E, generator=gen) * 3 + torch.linspace(-60, 60, T)[:, None]).to(dtype)
    dw, scale = torch.randn(T, k, generator=gen), 2.5
    r = L.gt_route(x.cuda(), k, score="sigmoid", renormalise=renormalise, scale=scale)
    got = L.gt_route_backward(dw.cuda(), x.cuda(), r.experts, score="sigmoid", renormalise=renormalise, scale=scale)

    chosen = r.experts.cpu().long()
    part, _ = ref.shares(x, chosen, "sigmoid", renormalise)
    rest = torch.sigmoid(-x.double().gather(1, chosen))
    g = scale * dw.double()
    mean = (part * g).sum(1, keepdim=True) if renormalise else 0.0
    value, size = torch.zeros(T, E, dtype=torch.float64), torch.zeros(T, E, dtype=torch.float64)
    value.scatter_(1, chosen, part * rest * (g - mean))
    most = (part * g.abs()).sum(1, keepdim=True) if renormalise else 0.0
    size.scatter_(1, chosen, part * rest * (g.abs() + most))
    # two exponentials, quotients and a sum of at most k terms in each share and in σ(−x), each
    # operation off by 2^-24 to 2^-23 of its value; the share's error counts in the mean too
    ref.check(got, ref.stored(value, size * (4 * k + 64) * ref.EPS + 2.0 ** -126, dtype), "dlogits")


def test_route_backward_against_differences(L):  # noqa: F811
    """The slope of a weight along its logit where the scores are within 1e-5 of 1: logits a quarter
    apart, so that the difference of two weights, far below them, comes from 64 bits."""
    x = torch.full((1, 4), 12.0)
    x[0] += torch.arange(4) / 4
    dw = torch.tensor([[1.0, 0.0, 0.0]])
    r = L.gt_route(x.cuda(), 3, score="sigmoid", renormalise=False)
    g = L.gt_route_backward(dw.cuda(), x.cuda(), r.experts, score="sigmoid", renormalise=False).cpu().double()
    h = 2.0 ** -7
    xs = x.double()
    top = int(r.experts[0, 0])
    s = [1 / (1 + math.exp(-(float(xs[0, top]) + sign * h))) for sign in (1, -1)]
    want = (s[0] - s[1]) / (2 * h)
    # the step's third-order term is h²/6 of the value, 1e-5; the difference keeps 2^-53 / 6e-8 of it
    assert abs(float(g[0, top]) - want) <= 2e-5 * want
