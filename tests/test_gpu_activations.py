"""The activations and their slopes in fp32 far into their tails, each value within 16 ulp of itself
(of the larger of its terms where they cancel), through every kernel that applies them."""
import math

import pytest
import torch

from test_gpu_layers import L  # noqa: F401

pytestmark = pytest.mark.gpu

REL = 16 * 2.0 ** -23
# rows: 3 go through the kernel of a few rows, 40 of 16 rows, 3000 through tiles
ROWS = [3, 40, 3000]


def points(name, M):
    lo, hi = {"silu": (-80.0, 20.0), "gelu": (-12.0, 8.0)}[name]   # (no value below fp32's normal ones)
    return torch.linspace(lo, hi, M, dtype=torch.float64).float()


def exact(name, x):
    """Value, slope, and the sum of the magnitudes of the slope's terms."""
    x = x.double()
    if name == "silu":
        s, rest = torch.sigmoid(x), torch.sigmoid(-x)
        return x * s, s + x * s * rest, s + x.abs() * s * rest
    cdf = 0.5 * torch.special.erfc(-x / math.sqrt(2))
    bell = torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    return x * cdf, cdf + x * bell, cdf + x.abs() * bell


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M", ROWS)
@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_values_and_slopes(L, name, M, gated):  # noqa: F811
    """X·W with one k and a W of ones: the pre-activations are X itself (the up values one)."""
    print(f"activation {name} {M} gated {gated}", flush=True)
    x, N = points(name, M), 8
    X = x.cuda().view(M, 1)
    W = torch.ones(1, N, device="cuda")
    ups = torch.zeros(2 * N, device="cuda")
    ups[N:] = 1
    if gated:
        W = torch.cat((W, torch.zeros(1, N, device="cuda")), dim=1)
    P = torch.empty(M, W.shape[1], device="cuda")
    Y = L.gt_linear(X, W, bias=ups if gated else None, act=name, gated=gated, P=P)
    assert torch.equal(P[:, :N], X.expand(M, N))
    value, slope, size = exact(name, x)
    assert bool(((Y.cpu().double() - value[:, None]).abs() <= REL * value.abs()[:, None]).all())

    # one output column at a time reaches dX, so that it holds one slope
    dY = torch.zeros(M, N, device="cuda")
    dY[:, 3] = 1
    dX, _, _ = L.gt_linear_backward(dY, X, W, P=P, act=name, gated=gated, need=("dX",), bias=False)
    assert bool(((dX.cpu().double()[:, 0] - slope).abs() <= REL * size).all())


@pytest.mark.parametrize("N", [72, 20])
@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_slopes_of_experts(L, name, N):  # noqa: F811
    """The same in the experts' hidden gradient: dH is one in one column, so dW1 is the slopes of one
    token."""
    x = points(name, N)
    r = L.gt_route(torch.zeros(1, 1, device="cuda"), 1)
    X, dY = torch.ones(1, 1, device="cuda"), torch.ones(1, 1, device="cuda")
    W1, W2 = x.cuda().view(1, 1, N), torch.ones(1, N, 1, device="cuda")
    P = torch.empty(1, N, device="cuda")
    L.gt_experts(X, r, W1, W2, act=name, P=P)
    assert torch.equal(P[0].cpu(), x)
    g = L.gt_experts_backward(dY, X, r, W1, W2, P, act=name)
    value, slope, size = exact(name, x)
    assert bool(((g.dW1[0, 0].cpu().double() - slope).abs() <= REL * size).all())
    assert bool(((g.dW2[0, :, 0].cpu().double() - value).abs() <= REL * value.abs()).all())
