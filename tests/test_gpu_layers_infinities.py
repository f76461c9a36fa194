"""Infinities and NaN at the end of a row, in every kernel that multiplies rows by a matrix: they
reach their own row alone, an infinity as an infinity."""
import math

import pytest
import torch

from test_gpu_layers import BF16, F32, IDS, L  # noqa: F401

pytestmark = pytest.mark.gpu

# rows: 1 … 4 a few rows, to 64 the kernel of 16 rows or tiles, above them tiles
ROWS = [1, 2, 3, 4, 5, 16, 40, 130]
# N, K: odd and even ends of a load, of a step and of a stage; narrow and long, in K slices
SIZES = [(72, 1), (72, 33), (64, 100), (129, 127), (264, 777), (64, 4100), (40, 4097), (72, 2088)]


def operands(dtype, M, N, K):
    gen = torch.Generator().manual_seed(M * N + K)
    X = torch.randint(-2, 3, (M, K), generator=gen).to(dtype).cuda()
    W = torch.randint(1, 3, (K, N), generator=gen)
    W[:, ::3] *= -1      # no zeros: an infinity is one in every column
    return X, W.to(dtype).cuda()


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("M", ROWS)
@pytest.mark.parametrize("dtype", [BF16, F32], ids=IDS.get)
def test_linear(L, dtype, M, size):  # noqa: F811
    N, K = size
    print(f"infinities {dtype} {M} {size}", flush=True)
    X, W = operands(dtype, M, N, K)
    clean = X.float() @ W.float()
    for row, value in ((M - 1, math.inf), (0, -math.inf)):
        X[row, K - 1] = value
        Y = L.gt_linear(X, W, Y=torch.empty(M, N, device="cuda"))
        want = clean.clone()
        want[row] = value * W[K - 1].float()
        assert torch.equal(Y, want), (row, value)
        X[row, K - 1] = math.nan
        Y = L.gt_linear(X, W, Y=torch.empty(M, N, device="cuda"))
        assert bool(Y[row].isnan().all())
        rest = [r for r in range(M) if r != row]
        assert torch.equal(Y[rest], clean[rest])
        X[row, K - 1] = 0
        clean = X.float() @ W.float()


@pytest.mark.parametrize("T,k", [(1, 2), (2, 1), (7, 2), (30, 2)])
@pytest.mark.parametrize("D,H", [(33, 40), (777, 72), (4100, 136)])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=IDS.get)
def test_experts(L, dtype, D, H, T, k):  # noqa: F811
    """A token that ends with an infinity: its pre-activations are infinite, the others' as before."""
    print(f"infinities of experts {dtype} {T} {k} {D} {H}", flush=True)
    E = 4
    gen = torch.Generator().manual_seed(T + D)
    r = L.gt_route(torch.randn(T, E, generator=gen).cuda(), k)
    X, _ = operands(dtype, T, 1, D)
    W1 = torch.stack([operands(dtype, e + 1, H, D)[1] for e in range(E)])
    W2 = torch.ones(E, H, D, dtype=dtype, device="cuda")
    P, Q = (torch.empty(T * k, H, dtype=dtype, device="cuda") for _ in range(2))
    Y = L.gt_experts(X, r, W1, W2, act="relu", P=P)
    X[T - 1, D - 1] = math.inf
    Z = L.gt_experts(X, r, W1, W2, act="relu", P=Q)
    place = r.place.long()
    for s in range(k):
        assert torch.equal(Q[place[T - 1, s]].float(), math.inf * W1[r.experts[T - 1, s], D - 1].float())
        assert torch.equal(Q[place[:T - 1, s]], P[place[:T - 1, s]])
    assert bool((Z[T - 1] == math.inf).all()) and torch.equal(Z[:T - 1], Y[:T - 1])
