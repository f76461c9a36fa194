"""The 8-bit products in every form (layers8_forms): whole numbers, which are exact on any path, the last
rounding being the only one; and values of any size, within bounds of the form that was taken."""
import itertools

import pytest
import torch

import layers8_plain as ref8
import layers_plain as ref
from layers8_forms import FORMS, TYPES, form_of
from layers_plain import EPS as E

pytestmark = pytest.mark.gpu

CODES = [(torch.float8_e4m3fn, torch.float8_e4m3fn), (torch.float8_e5m2, torch.float8_e4m3fn),
         (torch.float8_e4m3fn, torch.float8_e5m2), (torch.float8_e5m2, torch.float8_e5m2)]


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_1909_10616_amd import layers
    layers.lib()
    return layers


def among_nans(t):
    """The same codes, rows at 16-byte aligned addresses, NaN codes around them and behind each row."""
    M, K = t.shape
    buf = torch.full((M + 2, (K + 15) // 16 * 16 + 32), 0x7f, dtype=torch.uint8, device="cuda")
    view = buf[1:1 + M, 16:16 + K]
    view.copy_(t.view(torch.uint8))
    return view.view(t.dtype)


def scales_among_nans(s):
    buf = torch.full((s.shape[0] + 2, s.shape[1] + 3), float("nan"), device="cuda")
    view = buf[1:1 + s.shape[0], 1:1 + s.shape[1]]
    view.copy_(s)
    return view


class Out:
    """An output, perhaps with values, inside a larger one whose other elements have to stay."""

    def __init__(self, M, N, dtype, values=None):
        self.buf = torch.full((M + 2, N + 5), -77.0, dtype=dtype, device="cuda")
        self.view = self.buf[1:1 + M, :N]
        if values is not None:
            self.view.copy_(values)

    def untouched(self):
        self.view.fill_(-77.0)
        return bool((self.buf == -77.0).all())


def spread(s, rows, cols, block):
    s = s.double().repeat_interleave(128, dim=1)[:, :cols]
    return s.repeat_interleave(128, dim=0)[:rows] if block == "square" else s


def draws(seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return gen, lambda *s: torch.randn(*s, generator=gen, device="cuda")


@pytest.mark.parametrize("wblock", ["square", "row"])
@pytest.mark.parametrize("case", FORMS, ids=str)
def test_whole_numbers(L, case, wblock):
    """Codes up to 3 (products up to 9, sums of 8 of them up to 72: nothing 13 bits below the largest) with
    scales that are powers of two, a bias, relu and a residual that is the output, of whole numbers: the
    exact value rounded once to Y's type; gated, the fp32 product of two exact values, rounded again."""
    M, N, K, gated, out = case
    dtype, wide, kb = TYPES[out], N * (2 if gated else 1), -(-K // 128)
    for i, (xt, wt) in enumerate(CODES):
        if M * wide * K > 1 << 34 and i not in (0, 1 + (wblock == "row")):
            continue
        gen, _ = draws(i)
        ints = lambda most, *s: torch.randint(-most, most + 1, s, generator=gen, device="cuda").float()  # noqa: E731
        x, w = ints(3, M, K), ints(3, wide, K)
        sx, sw = 2.0 ** ints(1, M, kb), 2.0 ** ints(1, wide if wblock == "row" else ref8.blocks(wide), kb)
        X = L.Codes(among_nans(x.to(xt)), scales_among_nans(sx))
        W = L.Codes(among_nans(w.to(wt)), scales_among_nans(sw))
        bias = ints(4, wide).to(dtype) if i % 2 else None
        R = None if gated else ints(4, M, N).to(dtype)
        act = "relu" if i > 1 and not gated else "none"
        Y = Out(M, N, dtype, R)
        print(f"whole {case} {wblock} {xt} {wt}", flush=True)
        assert form_of(L, X, W, Y.view, gated)[0] == FORMS[case]
        L.gt_linear_fp8(X, W, bias=bias, residual=None if gated else Y.view, act=act, gated=gated, Y=Y.view)
        torch.cuda.synchronize()
        P = torch.mm(x.double() * spread(sx, M, K, "row"), (w.double() * spread(sw, wide, K, wblock)).t().contiguous())
        P = P if bias is None else P + bias.double()
        if gated:
            want = P[:, :N].float() * P[:, N:].float()
        else:
            want = ((P.clamp(min=0) if act == "relu" else P) + R.double()).float()
        assert torch.equal(Y.view, want.to(dtype)), int((Y.view != want.to(dtype)).sum())
        assert Y.untouched()


def dropped(a, b):
    """What the 8-bit instructions' sums may lose, for operands with their scales whose b has symmetric
    signs: of the 8 neighbouring products that they add at once, each loses what lies below 2^-13 of
    the largest, towards zero, so by less than u = 2^-13·(the largest) and with the sign of the product; the
    largest loses nothing. Given the magnitudes these are independent and symmetric: by Hoeffding's
    inequality their sum passes 8·√(7·Σu²) with a probability of 2·e^-32."""
    squares = torch.zeros(a.shape[0], b.shape[0], device="cuda")
    a, b = a.abs().float().t().contiguous(), b.abs().float().t().contiguous()
    for k in range(0, a.shape[0], 8):
        most = torch.zeros_like(squares)
        for j in range(k, min(k + 8, a.shape[0])):
            torch.maximum(most, torch.outer(a[j], b[j]), out=most)
        squares.addcmul_(most, most)
    return 8.001 * (7 * squares.double()).sqrt() * 2.0 ** -13


@pytest.mark.parametrize("wblock", ["square", "row"])
@pytest.mark.parametrize("case", FORMS, ids=str)
def test_values(L, case, wblock):
    """Sums in fp32 where few rows or an fp32 result make them so, the bound of 'dropped' beside that in tiles
    with a bf16 result."""
    M, N, K, gated, out = case
    dtype, wide = TYPES[out], N * (2 if gated else 1)
    act, i = ("silu", 1) if gated else ("gelu", 2) if K % 2 else ("none", 3)
    gen, normal = draws(K)
    size = torch.exp(normal(M, ref8.blocks(K))).repeat_interleave(128, 1)[:, :K]
    q = L.gt_quantise(normal(M, K) * size + 0.3, code=("e4m3", "e5m2")[i % 2]).codes
    p = L.gt_quantise(normal(wide, K) * K ** -0.5, block=wblock).codes
    X = L.Codes(among_nans(q.values), scales_among_nans(q.scales))
    W = L.Codes(among_nans(p.values), scales_among_nans(p.scales))
    bias, R, Y = normal(wide).to(dtype), normal(M, N).to(dtype), Out(M, N, dtype)
    print(f"values {case} {wblock} {act}", flush=True)
    took, fp32 = form_of(L, X, W, Y.view, gated)
    assert took == FORMS[case]
    L.gt_linear_fp8(X, W, bias=bias, residual=R, act=act, gated=gated, Y=Y.view)
    torch.cuda.synchronize()
    a = q.values.float().double() * spread(q.scales, M, K, "row")
    b = p.values.float().double() * spread(p.scales, wide, K, wblock)
    P = torch.mm(a, b.t().contiguous())
    # a block's 128 products and the blocks, a whole last place at each addition (layers8_plain.linear)
    dP = (2 * 128 + 2 * (ref8.blocks(K) + 12)) * E * torch.mm(a.abs(), b.abs().t().contiguous())
    if not fp32:
        dP = dP + dropped(a, b)
    P = P + bias.double()
    V, dV = ref.activate(P, dP + 2 * E * P.abs(), act, gated)
    V = V + R.double()
    V, dV = ref.stored(V, dV + 2 * E * V.abs(), dtype)
    off = (Y.view.double() - V).abs()
    assert bool((off <= dV).all()), (int((off > dV).sum()), float((off / dV).max()))
    assert Y.untouched()


def test_what_the_instructions_drop(L):
    """A term below 2^-13 of the largest of its 8 neighbouring products is dropped, of a larger one what lies below,
    towards zero; in another 8, in fp32, nothing. An fp32 result and the kernels of few rows keep it all."""
    seen = set()
    for M, dtype in itertools.product((1, 16, 1024), TYPES.values()):
        for small, sign in itertools.product((1, 2, 3, 4, 7, 8, 15), (1, -1)):
            for at, near in ((1, True), (7, True), (9, False), (900, False)):
                x, w = torch.zeros(M, 1024, device="cuda"), torch.zeros(1024, 1024, device="cuda")
                x[:, 0], x[:, 2], x[:, at] = 256, -256, sign * small
                w[:, 0] = w[:, 2] = 128
                w[:, at] = 1
                one = torch.ones(M, 8, device="cuda"), torch.ones(1024, 8, device="cuda")
                Y = torch.empty(M, 1024, dtype=dtype, device="cuda")
                X, W = L.Codes(x.to(torch.float8_e4m3fn), one[0]), L.Codes(w.to(torch.float8_e4m3fn), one[1])
                L.gt_linear_fp8(X, W, Y=Y)
                torch.cuda.synchronize()
                fp32 = form_of(L, X, W, Y, False)[1]
                assert fp32 or dtype is torch.bfloat16
                seen.add((dtype, fp32))
                want = small // 4 * 4 if near and not fp32 else small
                assert bool((Y == sign * want).all()), (M, dtype, small, sign, at)
    assert len(seen) == 3
