"""8-bit products whose blocks are summed in fp32 on request, whatever form they take and with a bf16
result: values within the fp32 bound, and outliers that cancel."""
import pytest
import torch

import layers8_plain as ref8
import layers_plain as ref
from layers8_forms import FORMS, form_of
from layers_plain import EPS as E
from test_gpu_layers8_forms import CODES, Out, among_nans, draws, scales_among_nans, spread

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
TILED = [c for c, (rows, _, _) in FORMS.items() if rows == 0 and c[4] == "bf16" and c[2] < 10000]


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_1909_10616_amd import layers
    layers.lib()
    return layers


@pytest.mark.parametrize("wblock", ["square", "row"])
@pytest.mark.parametrize("case", TILED, ids=str)
def test_values(L, case, wblock):
    """The bound of layers8_plain.linear with an fp32 result, and the one rounding to bf16."""
    M, N, K, gated, _ = case
    wide = N * (2 if gated else 1)
    act, i = ("silu", 1) if gated else ("gelu", 2) if K % 2 else ("none", 3)
    gen, normal = draws(K)
    q = L.gt_quantise(normal(M, K) + 0.3, code=("e4m3", "e5m2")[i % 2]).codes
    p = L.gt_quantise(normal(wide, K) * K ** -0.5, block=wblock).codes
    X = L.Codes(among_nans(q.values), scales_among_nans(q.scales))
    W = L.Codes(among_nans(p.values), scales_among_nans(p.scales))
    bias, R, Y = normal(wide).to(BF16), normal(M, N).to(BF16), Out(M, N, BF16)
    print(f"exact {case} {wblock}", flush=True)
    (rows, tile, _), fp32 = form_of(L, X, W, Y.view, gated, exact=1)
    assert fp32 and (rows > 0 or tile > 0)
    L.gt_linear_fp8(X, W, bias=bias, residual=R, act=act, gated=gated, Y=Y.view, exact=True)
    torch.cuda.synchronize()
    a = q.values.float().double() * spread(q.scales, M, K, "row")
    b = p.values.float().double() * spread(p.scales, wide, K, wblock)
    P = torch.mm(a, b.t().contiguous()) + bias.double()
    dP = (2 * 128 + 2 * (ref8.blocks(K) + 12)) * E * torch.mm(a.abs(), b.abs().t().contiguous())
    V, dV = ref.activate(P, dP + 2 * E * P.abs(), act, gated)
    V = V + R.double()
    V, dV = ref.stored(V, dV + 2 * E * V.abs(), BF16)
    off = (Y.view.double() - V).abs()
    assert bool((off <= dV).all()), (int((off > dV).sum()), float((off / dV).max()))
    assert Y.untouched()


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("shape", [(1, 1024, 1024), (130, 520, 333), (1024, 1024, 256), (2050, 2056, 333),
                                   (4096, 4096, 1000), (600, 2050, 5003)], ids=str)
def test_outliers_that_cancel(L, shape, gated):
    """2^15 and −2^15 among the same 8 products, 13 to 17 bits above the rest: whole numbers, exact in fp32 in any
    order (their magnitudes' sum is below 2^24)."""
    M, N, K = shape
    wide = 2 * N if gated else N
    for i, (xt, wt) in enumerate(CODES):
        gen, _ = draws(i)
        x = torch.randint(-1, 2, (M, K), generator=gen, device="cuda").float()
        w = torch.randint(-1, 2, (wide, K), generator=gen, device="cuda").float()
        at = torch.arange(0, K - K % 8, 104, device="cuda")
        x[:, at], x[:, at + 5] = 256.0, -256.0
        w[:, at] = w[:, at + 5] = 128.0
        # 2·2^15 at up to 49 places, and a few thousand of 1
        assert 2 * 2 ** 15 * len(at) + K < 1 << 24
        kb = -(-K // 128)
        X = L.Codes(among_nans(x.to(xt)), torch.ones(M, kb, device="cuda"))
        W = L.Codes(among_nans(w.to(wt)), torch.ones(wide, kb, device="cuda"))
        Y = Out(M, N, BF16)
        print(f"outliers {shape} gated {gated} {xt} {wt}", flush=True)
        L.gt_linear_fp8(X, W, gated=gated, Y=Y.view, exact=True)
        torch.cuda.synchronize()
        P = torch.mm(x.double(), w.double().t().contiguous()).float()
        want = P[:, :N] * P[:, N:] if gated else P
        assert torch.equal(Y.view, want.to(BF16))
        assert Y.untouched()


def test_an_fp32_result_is_so_anyway(L):
    gen, normal = draws(1)
    q, p = L.gt_quantise(normal(700, 900)).codes, L.gt_quantise(normal(500, 900), block="square").codes
    Y = [L.gt_linear_fp8(q, p, Y=torch.empty(700, 500, device="cuda"), exact=e) for e in (False, True)]
    torch.cuda.synchronize()
    assert torch.equal(*Y)
    few = [L.gt_linear_fp8(L.Codes(q.values[:2], q.scales[:2]), p, exact=e) for e in (False, True)]
    torch.cuda.synchronize()
    assert torch.equal(*few)
