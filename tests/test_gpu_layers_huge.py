"""Extents whose work-items, taken as a launch, would pass 2^32, and sums of almost 2^31 terms: a
quarter of a billion and more rows or columns of few values, whose results are known."""
import pytest
import torch

from test_gpu_layers import BF16, F32, L  # noqa: F401

pytestmark = pytest.mark.gpu

# 9·2^25 and what follows it: sums of ones of it, and of its parts, are whole in fp32 (and in bf16)
MANY = 9 << 25


def every(*conditions):
    """Whether all hold (outside the assertion, whose report would go through the tensors)."""
    return all(bool(c.all()) for c in conditions)


def ones(*shape, dtype=BF16):
    return torch.ones(*shape, dtype=dtype, device="cuda")


@pytest.fixture(autouse=True)
def free():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("M", [1, 4, 5])
def test_linear_of_many_columns(L, M):  # noqa: F811
    print(f"linear {M} x {MANY}", flush=True)
    W = ones(1, MANY)
    W[0, 1::2] = 2
    Y = L.gt_linear(ones(M, 1), W, bias=None)
    held = every(Y[:, ::2] == 1, Y[:, 1::2] == 2)
    assert held


def test_gated_linear_of_many_columns(L):  # noqa: F811
    W = ones(1, 2 * MANY)
    W[0, MANY:] = 3
    Y = L.gt_linear(ones(1, 1), W, gated=True)
    held = every(Y == 3)
    assert held


@pytest.mark.parametrize("K", [(1 << 31) - 8, (1 << 31) - 3])
def test_linear_of_a_long_sum(L, K):  # noqa: F811
    """The longest k there are: ones among zeros, the first and the last k among them."""
    X, W = torch.zeros(1, K, dtype=BF16, device="cuda"), ones(K, 4)
    at = torch.tensor([0, 1, 1 << 20, (1 << 30) + 7, K - 40, K - 33, K - 9, K - 1], device="cuda")
    X[0, at] = 1
    assert L.gt_linear(X, W).tolist() == [[8.0] * 4]


def test_linear_of_many_rows(L):  # noqa: F811
    X = ones(MANY, 1)
    X[1::2] = 2
    Y = L.gt_linear(X, ones(1, 1), act="relu")
    held = every(Y == X)
    assert held


@pytest.mark.parametrize("M,N", [(MANY, 1), (1, MANY), (2, MANY + 5)])
def test_linear_backward(L, M, N):  # noqa: F811
    print(f"linear_backward {M} x {N}", flush=True)
    dY, X, W = ones(M, N), ones(M, 1), ones(1, N)
    dX, dW, db = L.gt_linear_backward(dY, X, W, P=dY, act="relu")
    held = every(db == M, dW == M)
    assert held
    # (a sum of N ones, from partial sums that round at 2^-24 of themselves, stored in bf16)
    held = every((dX.double() - N).abs() <= N * 2.0 ** -7)
    assert held


@pytest.mark.parametrize("T,E,k", [(MANY, 2, 1), (70_000_001, 257, 1)])
def test_route_backward(L, T, E, k):  # noqa: F811
    print(f"route_backward {T} of {E}", flush=True)
    x = torch.zeros(T, E, dtype=BF16, device="cuda")
    experts = torch.zeros(T, k, dtype=torch.int32, device="cuda")
    d = L.gt_route_backward(ones(T, k, dtype=F32), x, experts, score="sigmoid", renormalise=False)
    held = every(d[:, 0] == 0.25, d[:, 1:] == 0)
    assert held


def test_experts_of_too_many_entries_are_refused(L):  # noqa: F811
    a = L.gt_experts_args(1 << 29, 8, 8, 4, 2, 1, 0, 256, 8, 256, 8, 64, 256, 8, 64, None, None, None, 8, 256, 8,
                          None, 8, 256, 256, 256, 256)
    with pytest.raises(L.gt.GemmTuneError, match="out of range"):
        L.workspace_bytes("gt_experts", a)
