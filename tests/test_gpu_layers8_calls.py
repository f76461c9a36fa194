"""Calls of the norm, the quantising and the 8-bit layers that their other tests do not make:
what the binding refuses, offsets past 32 bits, outputs that are inputs, a scratch of exactly
the size asked for, two streams at once, a training step inside a graph beside eager autograd."""
import math

import pytest
import torch

import layers8_plain as ref8
import layers_plain as ref
from test_gpu_layers8 import framed, nans, operands, rows

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_1909_10616_amd import layers
    layers.lib()
    return layers


def test_refusals(L):
    z = lambda *s, t=F32: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
    X, v = z(4, 256), z(4)
    q = L.gt_quantise(X).codes
    W = L.gt_quantise(z(64, 256), block="square").codes
    bad = [
        (lambda: L.gt_norm(z(4, 4, 4)), "2 dimensions"), (lambda: L.gt_norm(X.half()), "float32 or bfloat16"),
        (lambda: L.gt_norm(X, z(255)), "weight has shape"), (lambda: L.gt_norm(X, z(256, t=BF16)), "weight must be"),
        (lambda: L.gt_norm(X, z(256), z(256, t=BF16)), "bias must be"), (lambda: L.gt_norm(X, eps=-1.0), "eps"),
        (lambda: L.gt_norm(X, eps=math.nan), "eps"), (lambda: L.gt_norm(X, Y=z(4, 256, t=BF16)), "Y must be"),
        (lambda: L.gt_norm(X, mean=z(3)), "mean has shape"), (lambda: L.gt_norm(X, rstd=z(4, t=BF16)), "rstd must be"),
        (lambda: L.gt_norm(X.t()), "rows of X"), (lambda: L.gt_norm(X, z(512)[::2]), "contiguous"),
        (lambda: L.gt_norm_fp8(X, code="e3m4"), "unknown code"), (lambda: L.gt_norm_fp8(X, Y=z(4, 255)), "Y has shape"),
        (lambda: L.gt_norm_backward(z(4, 255), X, v, v), "dY has shape"),
        (lambda: L.gt_norm_backward(X, X, z(5), v), "mean has shape"),
        (lambda: L.gt_norm_backward(X, X, v, v, weight=z(256, t=BF16)), "weight must be"),
        (lambda: L.gt_norm_backward(X, X, v, v, residual=z(4, 256, t=BF16)), "residual must be"),
        (lambda: L.gt_norm_backward(X, X, v, v, dX=z(3, 256)), "dX has shape"),
        (lambda: L.gt_quantise(X, block="column"), "unknown block"), (lambda: L.gt_quantise(X, code="e8"), "unknown code"),
        (lambda: L.gt_quantise(X, need=()), "need is"), (lambda: L.gt_quantise(X, need=("rows",)), "need is"),
        (lambda: L.gt_quantise(X.half()), "float32 or bfloat16"), (lambda: L.gt_quantise(v), "2 dimensions"),
        (lambda: L.gt_linear_fp8(X, W), "Codes"), (lambda: L.gt_linear_fp8(q, L.Codes(W.values, z(65, 2))), "scales of W"),
        (lambda: L.gt_linear_fp8(q, L.Codes(W.values, z(64, 3))), "scales of W"),
        (lambda: L.gt_linear_fp8(L.Codes(X, q.scales), W), "float8"),
        (lambda: L.gt_linear_fp8(L.Codes(q.values[:, :255], q.scales), W), "W has shape|X has shape"),
        (lambda: L.gt_linear_fp8(q, W, bias=z(63)), "bias has shape"),
        (lambda: L.gt_linear_fp8(q, W, bias=z(64), residual=z(4, 64, t=BF16)), "residual must be"),
        (lambda: L.gt_linear_fp8(q, W, bias=z(64), Y=z(4, 64, t=BF16)), "Y must be"),
        (lambda: L.gt_linear_fp8(q, W, residual=z(4, 64, t=torch.float16)), "float32 or bfloat16"),
        (lambda: L.gt_linear_fp8(q, L.Codes(W.values[:63], W.scales), gated=True), "even number"),
        (lambda: L.gt_linear_fp8(q, W, act="tanh"), "unknown activation"),
        (lambda: L.gt_linear_fp8(q, W, Y=z(4, 64, t=F32).t().contiguous().t()), "rows of Y"),
        (lambda: L.gt_linear_fp8(L.Codes(q.values, q.scales.cpu()), W), "scales of X"),
    ]
    for f, why in bad:
        with pytest.raises(ValueError, match=why):
            f()
    Y = z(4, 64)
    with pytest.raises(Exception, match="same rows"):
        wide = z(4, 80)
        L.gt_linear_fp8(q, W, residual=wide[:, :64], Y=wide.view(-1)[:256].view(4, 64))
    assert L.gt_linear_fp8(q, W, residual=Y, Y=Y) is Y


def test_offsets_past_32_bits(L):
    """4.3 GB of codes and of values: the first, the last and rows beside 2^31 and 2^32 bytes."""
    M, K, N = 1052000, 4096, 128
    at = torch.tensor([0, 1, 524287, 524288, 524289, 1048575, 1048576, 1048577, M - 1])
    gen = torch.Generator().manual_seed(1)
    some = rows(gen, len(at), K, BF16)
    w, sw = ref8.quantise(torch.randn(N, K, generator=gen) / 64, "square", "e4m3")
    W = L.Codes(w.cuda(), sw.cuda())
    X = torch.zeros(M, K, dtype=BF16, device="cuda")
    X[at] = some.cuda()
    q = L.gt_quantise(X, need=("codes", "transposed"))
    torch.cuda.synchronize()
    want, scales = ref8.quantise(some, "row", "e4m3")
    assert ref8.same_codes(q.codes.values[at], want) and torch.equal(q.codes.scales[at].cpu(), scales)
    # the transpose: these columns, among zeros
    cols = q.transposed.values[:, at].t().float().cpu()
    ts = q.transposed.scales[:, at // 128].t().cpu()
    assert float((cols * ts - some.float()).abs().sub(2.0 ** -4 * some.float().abs() + 2.0 ** -10 * ts).max()) <= 0
    del cols, ts
    for out in (BF16, F32):
        Y = L.gt_linear_fp8(q.codes, W, Y=torch.empty(M, N, dtype=out, device="cuda"))
        torch.cuda.synchronize()
        ref.check(Y[at], ref8.linear(want, scales, w, sw, dtype=out), "Y")
        assert float(Y.float().abs().sum(1).gt(0).sum()) == len(at)
    mean, rstd = torch.empty(2, M, device="cuda")
    L.gt_norm(X, mean=mean, rstd=rstd, Y=X)
    torch.cuda.synchronize()
    ref.check(X[at], ref8.norm(some, None, None, 1e-5, BF16)[0], "norm")
    codes = L.gt_norm_fp8(X)
    g = L.gt_norm_backward(X, X, mean, rstd, need=("dX",), bias=False, dX=X)
    torch.cuda.synchronize()
    assert bool(torch.isfinite(g.dX[at]).all()) and not bool(codes.values[2].view(torch.uint8).any())


@pytest.mark.parametrize("case", [(256, 2048, 8192, False), (300, 520, 4099, False), (100, 1030, 5000, True),
                                  (1999, 700, 3457, False)], ids=str)
def test_scratch_of_exactly_the_size(L, case):
    """The scratch between two guards, its contents NaN before."""
    import ctypes
    M, N, K, gated = case
    wide = 2 * N if gated else N
    X, W = operands(L, 5, M, wide, K, "e4m3", "e4m3", "square", 5)
    Y = torch.empty(M, N, dtype=BF16, device="cuda")
    kb = -(-K // 128)
    a = L.gt_linear_fp8_args(M, N, K, 1, 19 if gated else 0, 1, 0, 0, 1, 128, 0, X.values.data_ptr(), X.values.stride(0),
                             X.scales.data_ptr(), X.scales.stride(0), W.values.data_ptr(), W.values.stride(0),
                             W.scales.data_ptr(), W.scales.stride(0), None, None, 0, Y.data_ptr(), N)
    assert X.scales.shape[1] == kb
    need = L.workspace_bytes("gt_linear_fp8", a)
    buf = torch.full((need + 512,), 0xff, dtype=torch.uint8, device="cuda")
    assert L.lib().gt_linear_fp8(ctypes.byref(a), buf.data_ptr() + 256, need, None) == 0
    torch.cuda.synchronize()
    assert bool((buf[:256] == 0xff).all()) and bool((buf[256 + need:] == 0xff).all())
    ref.check(Y, ref8.linear(*X, *W, act="silu" if gated else "none", gated=gated), "Y")


def test_rows_at_odd_addresses_are_exact(L):
    """Codes whose rows no 16-byte load serves, past the few rows: copied, the same bits as aligned ones."""
    for M, N, K in ((700, 900, 1000), (1500, 130, 2051), (90, 4096, 4095)):
        X, W = operands(L, 7, M, N, K, "e5m2", "e4m3", "row", 0)
        odd = L.gt_linear_fp8(L.Codes(nans(X.values.cpu(), 5), X.scales), L.Codes(nans(W.values.cpu(), 7), W.scales),
                              Y=torch.empty(M, N, device="cuda"))
        even = L.gt_linear_fp8(L.Codes(nans(X.values.cpu(), 32), X.scales), L.Codes(nans(W.values.cpu(), 32), W.scales),
                               Y=torch.empty(M, N, device="cuda"))
        torch.cuda.synchronize()
        want = ref8.linear(*X, *W, wblock="row", dtype=F32)
        ref.check(odd, want, "odd")
        ref.check(even, want, "even")


def test_two_streams_at_once(L):
    """Calls in flight on two streams, each with its own scratch, give what they give alone."""
    gen = torch.Generator().manual_seed(6)
    X = [rows(gen, 600, 1024, BF16).cuda() for _ in range(2)]
    W = L.gt_quantise(torch.randn(512, 1024, generator=gen).cuda() / 32, block="square").codes
    dY = torch.randn(600, 1024, generator=gen).to(BF16).cuda()

    def work(x):
        mean, rstd = torch.empty(2, 600, device="cuda")
        c = L.gt_norm_fp8(x, mean=mean, rstd=rstd)
        y = L.gt_linear_fp8(c, W, Y=torch.empty(600, 512, device="cuda"))
        return (y, *L.gt_norm_backward(dY, x, mean, rstd), *L.gt_quantise(x, need="transposed").transposed)

    alone = [work(x) for x in X]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in X]
    for _ in range(5):
        got = []
        for s, x in zip(streams, X):
            with torch.cuda.stream(s):
                got.append(work(x))
        torch.cuda.synchronize()
        for have, want in zip(got, alone):
            for a, b in zip(have, want):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


class Layer(torch.autograd.Function):
    """norm, 8-bit product and their gradients, as a user would tie them to autograd."""

    @staticmethod
    def forward(ctx, L, X, w, b, W):
        mean, rstd = torch.empty(2, X.shape[0], device=X.device)
        H = L.gt_norm(X, w, b, mean=mean, rstd=rstd)
        h, q = L.gt_quantise(H, need=("codes", "transposed")), L.gt_quantise(W, block="square", need=("codes", "transposed"))
        ctx.L, ctx.kept = L, (X, w, mean, rstd, h.transposed, q.transposed)
        return L.gt_linear_fp8(h.codes, q.codes, Y=torch.empty(X.shape[0], W.shape[0], device=X.device))

    @staticmethod
    def backward(ctx, dY):
        L, (X, w, mean, rstd, h, q) = ctx.L, ctx.kept
        d = L.gt_quantise(dY.contiguous(), code="e5m2", need=("codes", "transposed"))
        dH = L.gt_linear_fp8(d.codes, q, Y=torch.empty(X.shape, device=X.device))
        dW = L.gt_linear_fp8(d.transposed, h, Y=torch.empty(q.values.shape[::-1], device=X.device))
        g = L.gt_norm_backward(dH, X, mean, rstd, weight=w)
        return None, g.dX, g.dweight, g.dbias, dW


def test_a_training_step_from_autograd(L):
    """The gradients that autograd hands on are the calls', and near 64 bits': the same run under plain
    autograd, each operand off by half a step of its code at most."""
    gen = torch.Generator().manual_seed(8)
    M, D, N = 96, 384, 256
    X, w, b, W = (t.cuda().requires_grad_() for t in (torch.randn(M, D, generator=gen), 1 + 0.1 * torch.randn(D, generator=gen),
                                                     0.1 * torch.randn(D, generator=gen),
                                                     torch.randn(N, D, generator=gen) * D ** -0.5))
    c = torch.randn(M, N, generator=gen).cuda()
    Y = Layer.apply(L, X, w, b, W)
    Y.backward(c)
    torch.cuda.synchronize()
    x, wd, bd, Wd = (ref.d(t).requires_grad_() for t in (X, w, b, W))
    m = x.mean(1, keepdim=True)
    y = ((x - m) / torch.sqrt(((x - m) ** 2).mean(1, keepdim=True) + 1e-5) * wd + bd) @ Wd.T
    y.backward(ref.d(c))
    # two operands of a product, off by at most 2^-4 (e4m3) and 2^-3 (e5m2) of themselves
    for have, want, off in ((Y, y, 2 * 2.0 ** -4), (X.grad, x.grad, 3 * 2.0 ** -4), (w.grad, wd.grad, 3 * 2.0 ** -4),
                            (b.grad, bd.grad, 3 * 2.0 ** -4), (W.grad, Wd.grad, 3 * 2.0 ** -4)):
        assert float((ref.d(have) - ref.d(want)).norm()) <= off * float(ref.d(want).norm())


def test_strided_scales_and_slices(L):
    """Codes that are columns, at a block's border, and rows of larger ones, with their scales."""
    X, W = operands(L, 3, 300, 260, 1024, "e4m3", "e4m3", "row", 0)
    x = L.Codes(X.values[7:207, 256:900], X.scales[7:207, 2:8])
    w = L.Codes(W.values[4:204, 256:900], W.scales[4:204, 2:8])
    Y = L.gt_linear_fp8(x, w, Y=torch.empty(200, 200, device="cuda"))
    torch.cuda.synchronize()
    ref.check(Y, ref8.linear(*x, *w, wblock="row", dtype=F32), "Y")
    assert framed(torch.ones(2, 2), 3).shape == (2, 2)
