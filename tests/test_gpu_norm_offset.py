"""The norm of rows far from zero: what a row's mean has lost to rounding is not in its values."""
import math

import pytest
import torch

import layers8_plain as ref8
import layers_plain as ref
from layers_plain import EPS as E
from layers_plain import d
from test_gpu_layers8 import BF16, F32, IDS

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_1909_10616_amd import layers
    layers.lib()
    return layers


def centred(X, w, b, eps, dtype):
    """(Y, bound), (mean, bound), (rstd, bound) where the rounding of the mean is taken out again.

    The first mean is off by at most dm = g·mean|x|, g of a row's chain of sums. The deviations
    from it round by E of themselves, their own mean by g + 2E of their mean magnitude: e1, in which
    dm enters only with another factor g. A value's deviation is then off by e1 and two
    roundings. Σ(deviations²)/n less that mean's square is the variance up to g + 6E of the sum
    (the sum, the terms' roundings, the division) and what e1 changes in the square."""
    x = d(X)
    N = x.shape[1]
    mean = x.mean(1, keepdim=True)
    away = (x - mean).abs()
    var = (away ** 2).mean(1, keepdim=True)
    rstd = (var + eps) ** -0.5
    g = 2 * ref8.chain(N) * E
    dm = g * x.abs().mean(1, keepdim=True)
    e1 = (g + 2 * E) * (away.mean(1, keepdim=True) + dm)
    dvar = (g + 6 * E) * (var + dm ** 2) + 2 * dm * e1 + e1 ** 2
    t = dvar / (var + eps)
    assert float(t.max()) < 0.01
    drstd = 0.5 * t * (1 + t) + 4 * E
    w = d(w) if w is not None else torch.ones(N, dtype=torch.float64)
    b = d(b) if b is not None else torch.zeros(N, dtype=torch.float64)
    h = (x - mean) * rstd
    err = (w.abs() * rstd * (e1 + 2 * E * (away + dm + e1)) * (1 + drstd) + (w * h).abs() * (drstd + 3 * E)
           + 2 * E * ((w * h).abs() + b.abs()) + 2.0 ** -126)
    y = h * w + b
    return (ref.stored(y, err, dtype), (mean.squeeze(1), (e1 + 2 * E * mean.abs()).squeeze(1)),
            (rstd.squeeze(1), (drstd * rstd).squeeze(1)))


@pytest.mark.parametrize("N", [7, 300, 1000, 1500, 4000, 6000, 12000, 20000])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS.get)
def test_far_from_zero(L, dtype, N):
    """Means of up to 1e5 deviations (fp32; bf16, whose values lie 2^-8 apart, up to 100)."""
    gen = torch.Generator().manual_seed(N)
    for i, far in enumerate((0.0, 30.0, 1e3, 1e4, 1e5) if dtype is F32 else (0.0, 10.0, 100.0)):
        x = (torch.randn(5, N, generator=gen) + far).to(dtype)
        x[1] = (torch.randn(N, generator=gen) * 1e-3 - 1e-3 * far).to(dtype)
        X = x.cuda()
        w, b = (torch.randn(N, generator=gen).cuda(), torch.randn(N, generator=gen).cuda()) if i % 2 else (None, None)
        mean, rstd = torch.empty(2, 5, device="cuda")
        print(f"{dtype} {N} mean {far}", flush=True)
        Y = L.gt_norm(X, w, b, eps=1e-9, mean=mean, rstd=rstd)
        exact = torch.empty(5, N, dtype=dtype, device="cuda")
        codes = L.gt_norm_fp8(X, w, b, eps=1e-9, Y=exact)
        torch.cuda.synchronize()
        want, wmean, wrstd = centred(X, w, b, 1e-9, dtype)
        ref.check(Y, want, "Y")
        ref.check(exact, want, "Y beside its codes")
        ref.check(mean, wmean, "mean")
        ref.check(rstd, wrstd, "rstd")
        if dtype is F32:   # codes of the same values
            q, s = ref8.quantise(exact, "row", "e4m3")
            assert torch.equal(codes.scales.cpu(), s) and ref8.same_codes(codes.values, q)


@pytest.mark.parametrize("N", [1, 5, 77, 1000, 1500, 4000, 9000, 20000])
def test_constant_rows(L, N):
    """Of a constant row nothing is left: Y is b, within what E of its mean is beside √eps, the codes
    have b's scale, and a variance that rounds below zero is no NaN."""
    x = torch.tensor([7.25, -1e4 / 3, 1e30, 0.0, -3e-30]).unsqueeze(1).expand(5, N).contiguous()
    b = torch.linspace(-1, 1, N)
    b[0] = 1.0
    X = x.cuda()
    mean, rstd = torch.empty(2, 5, device="cuda")
    Y = L.gt_norm(X, None, b.cuda(), eps=1e-3, mean=mean, rstd=rstd)
    codes = L.gt_norm_fp8(X, None, b.cuda(), eps=1e-3)
    torch.cuda.synchronize()
    g = 2 * ref8.chain(N) * E
    # the first mean is off by g of it, the second by g of what is left and a rounding
    left = (g + 2 * E) * g * d(x[:, :1]).abs()
    off = left / math.sqrt(1e-3) + 2 * E * (1 + left / math.sqrt(1e-3))
    live = [0, 3, 4]
    assert bool(((Y.cpu().double() - b.double()).abs() <= off)[live].all())
    assert bool(((codes.scales[:, 0].cpu().double() * 448 - 1).abs() <= off[:, 0] + 2 * E)[live].all())
    assert bool(((mean.cpu().double() - d(x[:, 0])).abs() <= 2 * E * d(x[:, 0]).abs() + left[:, 0]).all())
    assert not bool(torch.isnan(Y).any()) and not bool(torch.isnan(rstd).any())
    # nothing beyond the last column counts among the values whose largest is the scale
    Y = torch.empty(5, N, device="cuda")
    codes = L.gt_norm_fp8(X, eps=1e-3, Y=Y)
    torch.cuda.synchronize()
    q, s = ref8.quantise(Y, "row", "e4m3")
    assert torch.equal(codes.scales.cpu(), s) and ref8.same_codes(codes.values, q)


def test_variance_past_the_largest_value(L):
    """Squares that overflow leave rstd 0 and Y = b, as the formula in fp32 has it, not NaN."""
    for N in (40, 700, 1500, 3000, 6000, 12000, 20000):
        x = torch.randn(3, N, generator=torch.Generator().manual_seed(N)) * 1e25 + 1e26
        b = torch.linspace(-1, 1, N)
        mean, rstd = torch.empty(2, 3, device="cuda")
        Y = L.gt_norm(x.cuda(), None, b.cuda(), mean=mean, rstd=rstd)
        torch.cuda.synchronize()
        assert not bool(rstd.any()) and torch.equal(Y.cpu(), b.expand(3, N))


def test_sums_that_are_not_finite(L):
    """An infinity leaves its row an infinite mean and no numbers; deviations whose sum overflows, where the
    values' does not, leave rstd 0 and Y = b."""
    for N in (24, 700, 1500, 3000, 6000, 12000, 20000):
        x = torch.randn(4, N, generator=torch.Generator().manual_seed(N))
        x[0, 5], x[1, N - 1] = math.inf, -math.inf
        x[2] = 0
        # octets of a wavefront's first lanes, whose sums meet two lanes apart first: −3.3e38, 3.3e38, 3.3e38
        x[2, :8], x[2, 8:24] = -3.3e38 / 8, 3.3e38 / 8
        b = torch.linspace(-1, 1, N)
        mean, rstd = torch.empty(2, 4, device="cuda")
        Y = L.gt_norm(x.cuda(), None, b.cuda(), mean=mean, rstd=rstd)
        torch.cuda.synchronize()
        assert mean[:2].tolist() == [math.inf, -math.inf]
        assert bool(torch.isnan(rstd[:2]).all()) and bool(torch.isnan(Y[:2]).all())
        assert rstd[2].item() == 0 and torch.equal(Y[2].cpu(), b)
        assert abs(mean[2].item() / (3.3e38 / N) - 1) < 2.0 ** -20
        assert bool(torch.isfinite(Y[3]).all())
