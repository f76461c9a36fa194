"""The layer operators on the GPU at sizes whose last large tiles are cut into K
slices and joined afterwards: small whole numbers, exact in any order of their sums."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_1909_10616_amd import layers
    layers.lib()
    return layers


def ints(gen, *shape, most=2):
    return torch.randint(-most, most + 1, shape, generator=gen).to(BF16).cuda()


def framed(dtype, rows, cols, ld):
    """An output inside a buffer whose rest is checked afterwards."""
    buf = torch.full((rows + 2, ld), -77.0, dtype=dtype, device="cuda")
    return buf, buf[1:1 + rows, :cols]


def untouched(buf, rows, cols):
    rest = torch.ones_like(buf, dtype=torch.bool)
    rest[1:1 + rows, :cols] = False
    assert bool((buf[rest] == -77.0).all())


@pytest.mark.parametrize("odd", [0, 5])
@pytest.mark.parametrize("gated", [False, True])
def test_linear(L, gated, odd):
    """bias, residual and pre-activations; products below 2^24 and P below 2^8 in bf16."""
    M, N, K = (4340, 2048 - odd, 1032) if gated else (4340, 4096 - odd, 1032)
    print(f"linear {M} {N} {K} gated {gated}", flush=True)
    gen = torch.Generator().manual_seed(M + odd)
    wide = 2 * N if gated else N
    X = ints(gen, M, K, most=1)
    X[:, ::2] = 0
    W, b, R = ints(gen, K, wide, most=1), ints(gen, wide), ints(gen, M, N, most=9)
    ybuf, Y = framed(F32, M, N, N + 8 + odd)
    pbuf, P = framed(BF16, M, wide, wide + 8 + odd)
    L.gt_linear(X, W, bias=b, residual=R, act="relu", gated=gated, Y=Y, P=P)
    p = X.float() @ W.float() + b.float()
    assert float(p.abs().max()) <= 256
    want = p[:, :N].relu() * p[:, N:] if gated else p.relu()
    assert torch.equal(Y, want + R.float())
    assert torch.equal(P.float(), p)
    untouched(ybuf, M, N)
    untouched(pbuf, M, wide)


@pytest.mark.parametrize("dtype,M,N,K,gated", [(F32, 1100, 1104, 2056, False), (F32, 1100, 1099, 2060, False),
                                               (F32, 1100, 560, 2056, True), (F32, 1100, 555, 2056, True),
                                               (F32, 2304, 2304, 520, False), (BF16, 1999, 2624, 3464, False),
                                               (BF16, 1999, 2621, 3464, False)])
def test_linear_smaller_tiles(L, dtype, M, N, K, gated):
    print(f"linear {dtype} {M} {N} {K} gated {gated}", flush=True)
    gen = torch.Generator().manual_seed(N)
    wide = 2 * N if gated else N
    X, W, R = (ints(gen, *shape, most=1).to(dtype) for shape in ((M, K), (K, wide), (M, N)))
    ybuf, Y = framed(F32, M, N, N + 3)
    pbuf, P = framed(F32 if dtype == F32 else BF16, M, wide, wide + 5)
    L.gt_linear(X, W, residual=R, act="relu", gated=gated, Y=Y, P=P)
    p = X.float() @ W.float()
    assert float(p.abs().max()) <= 256
    assert torch.equal(Y, (p[:, :N].relu() * p[:, N:] if gated else p.relu()) + R.float())
    assert torch.equal(P.float(), p)
    untouched(ybuf, M, N)
    untouched(pbuf, M, wide)


@pytest.mark.parametrize("K", [4096, 4091])
def test_linear_backward(L, K):
    M, N = 4340, 1040
    print(f"linear_backward {M} {N} {K}", flush=True)
    gen = torch.Generator().manual_seed(K)
    dY, W, X = ints(gen, M, N, most=1), ints(gen, K, N, most=1), ints(gen, M, K, most=1)
    buf, dX = framed(BF16, M, K, K + 11)
    L.gt_linear_backward(dY, X, W, act="none", dX=dX, need=("dX",), bias=False)
    want = dY.float() @ W.float().t().contiguous()
    assert torch.equal(dX.float(), want.to(BF16).float())
    untouched(buf, M, K)


@pytest.mark.parametrize("T,k,D,H", [(1700, 2, 4600, 1032), (4000, 1, 4096, 2056), (4000, 1, 4091, 2056)])
def test_experts(L, T, k, D, H):
    """One-hot tokens, weights of one half and small whole matrices; an expert without rows and
    tokens without experts."""
    E = 5
    print(f"experts {T} {E} {k} {D} {H}", flush=True)
    gen = torch.Generator().manual_seed(D)
    x = torch.randn(T, E, generator=gen)
    x[:, 2] = -math.inf
    x[torch.rand(T, generator=gen) < 0.02] = -math.inf
    r = L.gt_route(x.cuda(), k)
    r = r._replace(weights=torch.full_like(r.weights, 0.5))
    at = torch.randint(0, D, (T,), generator=gen).cuda()
    X = torch.zeros(T, D, dtype=BF16, device="cuda")
    X[torch.arange(T), at] = 2.0
    W1, W2 = ints(gen, E, D, H), ints(gen, E, H, D, most=1)
    P = torch.zeros(T * k, H, dtype=BF16, device="cuda")
    Y = L.gt_experts(X, r, W1, W2, act="relu", P=P)
    dY = ints(gen, T, D, most=2)
    dY[:, 8:] = 0      # dH, and dP = dH / 2 where P > 0, stay whole or halves below 2^7
    g = L.gt_experts_backward(dY, X, r, W1, W2, P, act="relu", bias=False)

    chosen, place = r.experts.long(), r.place.long()
    Yw, dXw = torch.zeros(T, D, device="cuda"), torch.zeros(T, D, device="cuda")
    for e in range(E):
        for s in range(k):
            t = (chosen[:, s] == e).nonzero().flatten()
            h = 2.0 * W1[e].float()[at[t]]
            assert torch.equal(P[place[t, s]].float(), h)
            Yw[t] += 0.5 * (h.relu() @ W2[e].float())
            dp = 0.5 * (dY[t].float() @ W2[e].float().t().contiguous()) * (h > 0)
            dXw[t] += dp @ W1[e].float().t().contiguous()
    assert torch.equal(Y, Yw.to(BF16))
    assert torch.equal(g.dX, dXw.to(BF16))
