"""The norm, the quantising and the 8-bit layers on the GPU against their plain forms
(layers8_plain): codes bit for bit, every other value within its own rounding bound; what lies
around the operands is NaN and must not be read into a result, what lies around the outputs
must stay as it was."""
import itertools
import math

import pytest
import torch

import layers8_plain as ref8
import layers_plain as ref
from test_gpu_layers import Frame, note

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
IDS = {BF16: "bf16", F32: "f32", E4M3: "e4m3", E5M2: "e5m2"}


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_1909_10616_amd import layers
    layers.lib()
    return layers


def rows(gen, M, N, dtype=F32):
    """Values of sizes that differ from block to block."""
    size = torch.exp(2 * torch.randn(M, -(-N // 64), generator=gen)).repeat_interleave(64, 1)[:, :N]
    return (torch.randn(M, N, generator=gen) * size + 0.5).to(dtype)


def nans(t, pad):
    """The same codes inside a larger matrix of NaN codes; pad 32: rows at 16-byte aligned addresses."""
    if not pad:
        return t.cuda()
    ld = t.shape[1] + pad if pad != 32 else (t.shape[1] + 15) // 16 * 16 + pad
    buf = torch.full((t.shape[0] + 2, ld), 0x7f, dtype=torch.uint8, device="cuda")
    view = buf[1:1 + t.shape[0], pad // 2:pad // 2 + t.shape[1]]
    view.copy_(t.view(torch.uint8))
    return view.view(t.dtype)


def framed(t, pad):
    if not pad:
        return t.cuda()
    buf = torch.full((t.shape[0] + 2, t.shape[1] + pad), math.nan, device="cuda")
    view = buf[1:1 + t.shape[0], :t.shape[1]]
    view.copy_(t)
    return view


# ---------------------------------------------------------------------------
# quantise
# ---------------------------------------------------------------------------

QSHAPES = [(1, 1), (1, 128), (1, 129), (128, 1), (3, 7), (127, 255), (128, 128), (129, 130), (130, 1021), (257, 384),
           (5, 4096)]


@pytest.mark.parametrize("pow2", [False, True])
@pytest.mark.parametrize("code", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=IDS.get)
def test_quantise(L, dtype, code, pow2):
    for i, (M, N) in enumerate(QSHAPES):
        for block, pad in itertools.product(("row", "square"), (0, 5)):
            note(f"quantise {M}x{N} {block} pad {pad}")
            f = Frame(i, pad)
            x = rows(torch.Generator().manual_seed(i), M, N, dtype)
            X = f.place(x)
            got = L.gt_quantise(X, block=block, code=code, pow2=pow2, need=("codes", "transposed"))
            torch.cuda.synchronize()
            for have, v in zip(got, (x, x.T)):
                q, s = ref8.quantise(v, block, code, pow2)
                assert torch.equal(have.scales.cpu(), s)
                assert ref8.same_codes(have.values, q)
            one = L.gt_quantise(X, block=block, code=code, pow2=pow2)
            other = L.gt_quantise(X, block=block, code=code, pow2=pow2, need="transposed")
            assert one.transposed is None and other.codes is None
            for a, b in ((one.codes, got.codes), (other.transposed, got.transposed)):
                assert torch.equal(a.scales, b.scales)
                assert torch.equal(a.values.view(torch.uint8), b.values.view(torch.uint8))


@pytest.mark.parametrize("block", ["row", "square"])
@pytest.mark.parametrize("code", ["e4m3", "e5m2"])
def test_quantise_special_values(L, code, block):
    """Zeros, the smallest and largest magnitudes, halves between codes, NaN, infinities."""
    x = torch.zeros(130, 400)
    x[1, :128] = 2.0 ** -140                      # every value subnormal
    x[2, :128] = torch.linspace(-3.4e38, 3.4e38, 128)
    x[3, 128:256] = torch.arange(128) * 2.0 ** -130
    x[4, :128] = torch.arange(128) - 64.0
    x[4, 0] = ref8.LARGEST[ref8.FP8[code]]        # scale 1: codes and halves between them
    x[4, 64:128] = 1 + torch.arange(64) / 32.0
    x[5, 7] = math.nan
    x[5, 8] = 3.0
    x[129, 399] = math.inf
    x[129, 398] = 5.0
    x[128, 256:] = math.nan
    got = L.gt_quantise(x.cuda(), block=block, code=code, need=("codes", "transposed"))
    torch.cuda.synchronize()
    for have, v in zip(got, (x, x.T)):
        q, s = ref8.quantise(v, block, code)
        assert torch.equal(have.scales.cpu(), s)
        assert ref8.same_codes(have.values, q)


def test_quantise_writes_only_its_codes(L):
    """Through the C entry: rows and scales inside larger arrays, neighbours untouched."""
    import ctypes
    M, N = 131, 261
    x = rows(torch.Generator().manual_seed(3), M, N)
    X = x.cuda()
    for block, rows_of in (("row", (M, N)), ("square", (2, 3))):
        q = torch.full((M + 2, N + 11), 99, dtype=torch.uint8, device="cuda")
        t = torch.full((N + 2, M + 7), 99, dtype=torch.uint8, device="cuda")
        s = torch.full((rows_of[0] + 2, 3 + 2), -9.0, device="cuda")
        st = torch.full((rows_of[1] + 2, 2 + 2), -9.0, device="cuda")
        a = L.gt_quantise_args(M, N, 0, 0, L.BLOCKS[block], 0, X.data_ptr(), N, q[1:].data_ptr() + 3, N + 11,
                               s[1:].data_ptr() + 4, 5, t[1:].data_ptr() + 3, M + 7, st[1:].data_ptr() + 4, 4)
        assert L.lib().gt_quantise(ctypes.byref(a), None) == 0
        torch.cuda.synchronize()
        for buf, sc, v, (m, n) in ((q, s, x, (M, N)), (t, st, x.T, (N, M))):
            want, ws = ref8.quantise(v, block, "e4m3")
            assert torch.equal(buf[1:1 + m, 3:3 + n].cpu(), want.view(torch.uint8))
            assert torch.equal(sc[1:-1, 1:1 + ws.shape[1]].cpu(), ws)
            buf[1:1 + m, 3:3 + n] = 99
            sc[1:-1, 1:1 + ws.shape[1]] = -9.0
            assert bool((buf == 99).all()) and bool((sc == -9.0).all())


# ---------------------------------------------------------------------------
# norm
# ---------------------------------------------------------------------------

# widths that end inside an octet, a thread's octets, a workgroup's, and rows read in passes
NSHAPES = [(1, 1), (2, 7), (5, 8), (9, 512), (7, 513), (3, 1021), (4, 1024), (6, 2047), (5, 2049), (3, 4096), (2, 4104),
           (3, 8192), (2, 8199), (2, 16384), (2, 16385), (3, 33001), (700, 72), (2100, 40)]


@pytest.mark.parametrize("shape", NSHAPES, ids=str)
@pytest.mark.parametrize("dtype", [BF16, F32], ids=IDS.get)
def test_norm(L, dtype, shape):
    M, N = shape
    for i, (pad, kind) in enumerate(itertools.product((0, 5), ("both", "f32", "none"))):
        f = Frame(i, pad)
        X = f.place(rows(f.gen, M, N, dtype))
        wt = F32 if kind == "f32" else dtype
        w, b = (None, None) if kind == "none" else (f.normal(wt, N), f.normal(wt, N))
        eps = (1e-5, 0.1, 1e-6)[i % 3]
        mean, rstd = torch.empty(2, M, device="cuda")
        Y = f.output(dtype, M, N)
        note(f"norm {dtype} {shape} pad {pad} {kind}")
        assert L.gt_norm(X, w, b, eps=eps, Y=Y, mean=mean, rstd=rstd) is Y
        codes = L.gt_norm_fp8(X, w, b, eps=eps, code=("e4m3", "e5m2")[i % 2], pow2=i == 4)
        exact = f.output(F32, M, N) if dtype is F32 else None
        again = L.gt_norm_fp8(X, w, b, eps=eps, code=("e4m3", "e5m2")[i % 2], pow2=i == 4, Y=exact)
        torch.cuda.synchronize()
        want, wmean, wrstd = ref8.norm(X, w, b, eps, dtype)
        ref.check(Y, want, "Y")
        ref.check(mean, wmean, "mean")
        ref.check(rstd, wrstd, "rstd")
        f.untouched()
        assert torch.equal(codes.scales, again.scales)
        assert torch.equal(codes.values.view(torch.uint8), again.values.view(torch.uint8))
        if exact is not None:   # the codes are those of the unrounded values
            q, s = ref8.quantise(exact, "row", ("e4m3", "e5m2")[i % 2], i == 4)
            assert torch.equal(codes.scales.cpu(), s) and ref8.same_codes(codes.values, q)
        else:
            (y, err), _, _ = ref8.norm(X, w, b, eps, None)
            s = ref8.widen(codes.scales.cpu().double(), M, N, "row")
            near = {E4M3: (2.0 ** -4, 2.0 ** -10), E5M2: (2.0 ** -3, 2.0 ** -17)}[codes.values.dtype]
            off = (codes.values.cpu().float().double() * s - y).abs()
            # half a step of the code: relative, or of the smallest subnormal's step
            assert bool((off <= 1.001 * (near[0] * y.abs() + near[1] * s + err)).all())


def test_norm_far_from_zero_and_constant_rows(L):
    """A mean of many deviations costs no digits of them; a constant row has none."""
    gen = torch.Generator().manual_seed(1)
    for N in (300, 1500, 4000, 12000, 20000):
        x = torch.randint(-8, 9, (4, N), generator=gen).float() + 4096.0
        x[3] = 7.25
        X = x.cuda()
        Y = L.gt_norm(X, eps=1e-3)
        torch.cuda.synchronize()
        want, _, _ = ref8.norm(X, None, None, 1e-3, F32)
        ref.check(Y[:3], (want[0][:3], want[1][:3]), "Y")
        mean = x.double().mean(1)   # sums of whole numbers below 2^24·8 … are near; 7.25·N is exact
        assert float((Y[3].cpu().double() - (7.25 - mean[3]) / math.sqrt(1e-3)).abs().max()) <= 7.25 * 2.0 ** -22 / math.sqrt(1e-3)


def test_norm_in_place_and_nan_rows(L):
    for dtype, N in itertools.product((BF16, F32), (77, 4096, 20000)):
        x = rows(torch.Generator().manual_seed(N), 6, N, dtype)
        x[1, 5] = math.nan
        x[2, N - 1] = math.inf
        X = x.cuda()
        want = L.gt_norm(X)
        got = L.gt_norm(X, Y=X)
        torch.cuda.synchronize()
        assert got is X and torch.equal(torch.isnan(want), torch.isnan(X))
        assert bool(torch.isnan(X[1:3]).all()) and not bool(torch.isnan(X[[0, 3, 4, 5]]).any())
        live = [0, 3, 4, 5]
        assert torch.equal(X[live], want[live])


@pytest.mark.parametrize("shape", NSHAPES, ids=str)
@pytest.mark.parametrize("dtype", [BF16, F32], ids=IDS.get)
def test_norm_backward(L, dtype, shape):
    M, N = shape
    for i, (pad, kind) in enumerate(itertools.product((0, 5), ("both", "f32", "none"))):
        f = Frame(10 + i, pad)
        X, dY = f.place(rows(f.gen, M, N, dtype)), f.normal(dtype, M, N)
        w = None if kind == "none" else f.normal(F32 if kind == "f32" else dtype, N)
        R = f.normal(dtype, M, N) if i % 2 else None
        dX = f.output(dtype, M, N)
        mean, rstd = torch.empty(2, M, device="cuda")
        L.gt_norm(X, w, mean=mean, rstd=rstd)
        note(f"norm backward {dtype} {shape} pad {pad} {kind}")
        g = L.gt_norm_backward(dY, X, mean, rstd, weight=w, residual=R, dX=dX)
        torch.cuda.synchronize()
        assert g.dX is dX
        want = ref8.norm_backward(dY, X, mean, rstd, w, R, dtype)
        for have, (v, err), name in zip(g, want, ("dX", "dw", "db")):
            ref.check(have, (v, err), name)
        f.untouched()
        # each output alone, and in place of the residual or of dY
        assert torch.equal(L.gt_norm_backward(dY, X, mean, rstd, weight=w, need=("dweight",), bias=False).dweight, g.dweight)
        assert torch.equal(L.gt_norm_backward(dY, X, mean, rstd, weight=w, need=()).dbias, g.dbias)
        alone = L.gt_norm_backward(dY, X, mean, rstd, weight=w, residual=R, need="dX", bias=False)
        assert torch.equal(alone.dX, g.dX) and alone.dweight is None and alone.dbias is None
        into = R if R is not None else dY
        both = L.gt_norm_backward(dY, X, mean, rstd, weight=w, residual=R, dX=into)
        torch.cuda.synchronize()
        assert torch.equal(both.dX, g.dX) and torch.equal(both.dweight, g.dweight)


@pytest.mark.parametrize("shape", [(1024, 40), (1025, 40), (1023, 2056), (1040, 1000), (1030, 2050), (1026, 4100),
                                   (512, 4104), (513, 8200)], ids=str)
@pytest.mark.parametrize("dtype", [BF16, F32], ids=IDS.get)
def test_norm_backward_past_few_rows(L, dtype, shape):
    """Either side of the rows up to which one launch takes the columns' sums."""
    M, N = shape
    f = Frame(5, 3 if M % 2 else 8)   # (odd and aligned rows)
    X, dY = f.place(rows(f.gen, M, N, dtype)), f.normal(dtype, M, N)
    w = f.normal(F32, N)
    dX = f.output(dtype, M, N)
    mean, rstd = torch.empty(2, M, device="cuda")
    L.gt_norm(X, w, mean=mean, rstd=rstd)
    note(f"norm backward {dtype} {shape}")
    g = L.gt_norm_backward(dY, X, mean, rstd, weight=w, dX=dX)
    torch.cuda.synchronize()
    want = ref8.norm_backward(dY, X, mean, rstd, w, None, dtype)
    for have, (v, err), name in zip(g, want, ("dX", "dw", "db")):
        ref.check(have, (v, err), name)
    f.untouched()
    alone = L.gt_norm_backward(dY, X, mean, rstd, weight=w, need=("dweight",), bias=False)
    assert torch.equal(alone.dweight, g.dweight)
    both = L.gt_norm_backward(dY, X, mean, rstd, weight=w, dX=dY)
    torch.cuda.synchronize()
    assert torch.equal(both.dX, g.dX) and torch.equal(both.dweight, g.dweight) and torch.equal(both.dbias, g.dbias)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=IDS.get)
def test_norm_backward_where_dx_lies(L, dtype):
    """dX over all of dY, in the other columns of dY's rows, and over X: the sums are of what was there."""
    M, N = 300, 520
    gen = torch.Generator().manual_seed(2)
    x, y = rows(gen, M, N, dtype).cuda(), rows(gen, M, N, dtype).cuda()
    mean, rstd = torch.empty(2, M, device="cuda")
    L.gt_norm(x, mean=mean, rstd=rstd)
    want = L.gt_norm_backward(y, x, mean, rstd)
    wide = torch.empty(M, 2 * N, dtype=dtype, device="cuda")
    wide[:, :N] = y
    over, beside, X = y.clone(), wide[:, N:], x.clone()
    got = [L.gt_norm_backward(over, x, mean, rstd, dX=over), L.gt_norm_backward(wide[:, :N], x, mean, rstd, dX=beside),
           L.gt_norm_backward(y, X, mean, rstd, dX=X)]
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))
    assert torch.equal(wide[:, :N], y)


def test_norm_gradients_against_differences(L):
    """The directional derivative of Σ c·Y by central differences in 64 bits."""
    gen = torch.Generator().manual_seed(4)
    M, N = 5, 300
    x, c, w, b = (torch.randn(*s, generator=gen, dtype=torch.float64) for s in ((M, N), (M, N), (N,), (N,)))

    def loss(x, w, b):
        m = x.mean(1, keepdim=True)
        v = ((x - m) ** 2).mean(1, keepdim=True)
        return float((c * ((x - m) / torch.sqrt(v + 1e-2) * w + b)).sum())

    X, W = x.float().cuda(), w.float().cuda()
    mean, rstd = torch.empty(2, M, device="cuda")
    L.gt_norm(X, W, b.float().cuda(), eps=1e-2, mean=mean, rstd=rstd)
    g = L.gt_norm_backward(c.float().cuda(), X, mean, rstd, weight=W)
    torch.cuda.synchronize()
    for i, grad in enumerate(g):
        args = [x, w, b]
        step = torch.randn(args[i].shape, generator=gen, dtype=torch.float64)
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + 1e-5 * step, args[i] - 1e-5 * step
        want = (loss(*up) - loss(*down)) / 2e-5
        have = float((grad.cpu().double() * step).sum())
        # inputs rounded to fp32 (2^-24 of 1500 terms of order 1) and the differences' 1e-10·third derivative
        assert abs(have - want) <= 2e-3 * (1 + abs(want)), (i, have, want)


# ---------------------------------------------------------------------------
# linear of codes
# ---------------------------------------------------------------------------

SHAPES = [(1, 1, 1), (1, 64, 128), (1, 133, 1), (2, 16, 129), (3, 130, 77), (16, 128, 256), (17, 136, 200), (33, 64, 640),
          (64, 257, 1021), (65, 72, 24), (130, 131, 129), (129, 257, 400), (250, 264, 512), (257, 300, 1100)]


def operands(L, seed, M, wide, K, xcode, wcode, wblock, pad, xblock="row"):
    gen = torch.Generator().manual_seed(seed)
    x, sx = ref8.quantise(rows(gen, M, K), xblock, xcode)
    w, sw = ref8.quantise(rows(gen, wide, K) * K ** -0.5, wblock, wcode)
    return L.Codes(nans(x, pad), framed(sx, pad)), L.Codes(nans(w, pad), framed(sw, pad))


@pytest.mark.parametrize("pad", [0, 32, 5])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_linear_fp8(L, shape, pad):
    M, N, K = shape
    for i, (act, gated) in enumerate(itertools.product(("none", "relu", "gelu", "silu"), (False, True))):
        f = Frame(i, pad)
        wide = N * (2 if gated else 1)
        dtype = (BF16, F32)[i // 2 % 2]
        xcode, wcode = (("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2"))[(i + pad) % 4]
        wblock, xblock = ("square", "row")[(i + pad) // 2 % 2], ("row", "row", "row", "square")[i % 4]
        note(f"linear fp8 {shape} pad {pad} {act} gated {gated} {xcode}/{xblock} {wcode}/{wblock} {dtype}")
        X, W = operands(L, i, M, wide, K, xcode, wcode, wblock, pad, xblock)
        bias = f.normal(dtype, wide) if i % 3 else None
        R = f.normal(dtype, M, N) if i % 2 else None
        Y = f.output(F32 if i == 4 else dtype, M, N)
        assert L.gt_linear_fp8(X, W, bias=bias, residual=R, act=act, gated=gated, Y=Y) is Y
        torch.cuda.synchronize()
        ref.check(Y, ref8.linear(*X, *W, xblock, wblock, bias, R, act, gated, Y.dtype), "Y")
        f.untouched()


def whole(gen, rows_, cols, most, dtype):
    return torch.randint(-most, most + 1, (rows_, cols), generator=gen).float().to(dtype)


# every form and tile, K of a few blocks to many, sizes past the largest tile
LARGE = [(1, 4096, 4096), (4, 1024, 11008), (64, 4096, 2048), (100, 520, 8200), (520, 768, 320), (515, 1021, 333),
         (1030, 1032, 200), (2050, 2056, 136), (1024, 4104, 1000), (4100, 260, 512), (300, 2050, 4000)]


@pytest.mark.parametrize("wblock", ["square", "row"])
@pytest.mark.parametrize("case", LARGE, ids=str)
def test_linear_fp8_whole_numbers(L, case, wblock):
    """Small whole numbers with scales that are powers of two are exact in fp32, in any order and on any path."""
    M, N, K = case
    for i, gated in enumerate((False, True)):
        gen = torch.Generator().manual_seed(i)
        wide = N * (2 if gated else 1)
        x, w = whole(gen, M, K, 3, E4M3), whole(gen, wide, K, 3, (E4M3, E5M2)[i])
        kb = -(-K // 128)
        sx = 2.0 ** torch.randint(-1, 2, (M, kb), generator=gen).float()
        sw = 2.0 ** torch.randint(-1, 2, (wide if wblock == "row" else -(-wide // 128), kb), generator=gen).float()
        R = torch.randint(-4, 5, (M, N), generator=gen).float().cuda()
        note(f"whole {case} {wblock} gated {gated}")
        X, W = L.Codes(x.cuda(), sx.cuda()), L.Codes(w.cuda(), sw.cuda())
        Y = R.clone()
        got = L.gt_linear_fp8(X, W, residual=None if gated else Y, gated=gated, Y=Y)
        torch.cuda.synchronize()
        a = (x.float() * ref8.widen(sx, M, K, "row")).cuda().double()
        b = (w.float() * ref8.widen(sw, wide, K, wblock)).cuda().double()
        P = torch.mm(a, b.t().contiguous())
        if not gated:
            assert got is Y and torch.equal(Y.double(), P + R)
        else:   # two exact values' product, rounded once
            assert torch.equal(Y, P[:, :N].float() * P[:, N:].float())


def test_linear_fp8_zero_rows(L):
    X, W = operands(L, 0, 4, 64, 128, "e4m3", "e4m3", "square", 0)
    Y = L.gt_linear_fp8(L.Codes(X.values[:0], X.scales[:0]), W)
    assert Y.shape == (0, 64)
    assert L.gt_norm(torch.empty(0, 64, device="cuda")).shape == (0, 64)
    q = L.gt_quantise(torch.empty(0, 64, device="cuda"), need=("codes", "transposed"))
    assert q.codes.values.shape == (0, 64) and q.transposed.scales.shape == (64, 0)
    e = torch.empty(0, device="cuda")
    g = L.gt_norm_backward(torch.empty(0, 64, device="cuda"), torch.empty(0, 64, device="cuda"), e, e)
    torch.cuda.synchronize()
    assert g.dX.shape == (0, 64) and not g.dweight.any() and not g.dbias.any()


def test_linear_fp8_special_codes(L):
    """A NaN code, or an infinite scale with a zero code, is its row's NaN alone."""
    for M, N, K in ((3, 40, 300), (200, 300, 300), (300, 600, 700)):
        X, W = operands(L, 3, M, N, K, "e4m3", "e4m3", "row", 0)
        x = X.values.view(torch.uint8).clone()
        x[1, K - 1] = 0x7f
        s = W.scales.clone()
        w = W.values.view(torch.uint8).clone()
        s[7, 1] = math.inf
        w[7, 128:256] = 0
        clean = L.gt_linear_fp8(X, W)
        Y = L.gt_linear_fp8(L.Codes(x.view(E4M3), X.scales), L.Codes(w.view(E4M3), s))
        torch.cuda.synchronize()
        bad = torch.zeros(M, N, dtype=torch.bool)
        bad[1] = True
        bad[:, 7] = True
        assert torch.equal(torch.isnan(Y).cpu(), bad)
        assert torch.equal(Y[~bad.cuda()], clean[~bad.cuda()])


# ---------------------------------------------------------------------------
# together, streams, graphs
# ---------------------------------------------------------------------------

def block(L, X, w, b, W, dY):
    """A pre-norm residual layer Y = X + norm(X)·Wᵀ with 8-bit products, and its gradients: the run that
    a training step makes."""
    M = X.shape[0]
    mean, rstd = torch.empty(2, M, device=X.device)
    codes = L.gt_norm_fp8(X, w, b, mean=mean, rstd=rstd)
    wq = L.gt_quantise(W, block="square", need=("codes", "transposed"))
    Y = L.gt_linear_fp8(codes, wq.codes, residual=X)
    dq = L.gt_quantise(dY, code="e5m2", need=("codes", "transposed"))
    dH = L.gt_linear_fp8(dq.codes, wq.transposed)
    H = L.gt_norm(X, w, b)
    hq = L.gt_quantise(H, need="transposed").transposed
    dW = L.gt_linear_fp8(dq.transposed, hq, Y=torch.empty(W.shape, device=X.device))
    g = L.gt_norm_backward(dH, X, mean, rstd, weight=w, residual=dY)
    return Y, g.dX, dW, g.dweight, g.dbias


@pytest.mark.parametrize("M", [1, 130, 512])
def test_a_layer_together(L, M):
    """Forward and gradients of a pre-norm layer: against the same steps in plain form on the
    8-bit values that the calls made, and near the layer in 64 bits."""
    D = 256
    gen = torch.Generator().manual_seed(M)
    X, dY = rows(gen, M, D, BF16).cuda(), torch.randn(M, D, generator=gen).to(BF16).cuda()
    w, b = torch.randn(D, generator=gen).cuda(), torch.randn(D, generator=gen).cuda()
    W = (torch.randn(D, D, generator=gen) * D ** -0.5).to(BF16).cuda()
    Y, dX, dW, dw, db = block(L, X, w, b, W, dY)
    torch.cuda.synchronize()
    x, wd, bd, Wd = (ref.d(t).requires_grad_() for t in (X, w, b, W))
    m = x.mean(1, keepdim=True)
    h = (x - m) / torch.sqrt(((x - m) ** 2).mean(1, keepdim=True) + 1e-5) * wd + bd
    out = x + h @ Wd.T
    out.backward(ref.d(dY))
    # each operand is off by at most half a step of its code: e4m3 2^-4 and e5m2 2^-3 of itself. Of a
    # product's norm two such operands take at most their sum of the magnitudes' product; in 2-norm
    # over independent roundings far less. What is asked is that bound on norms.
    for have, want, off in ((Y - X, out.detach() - x.detach(), 2 * 2.0 ** -4), (dW, Wd.grad, 2.0 ** -4 + 2.0 ** -3),
                            (db, bd.grad, 2.0 ** -4 + 2.0 ** -3), (dw, wd.grad, 2.0 ** -4 + 2.0 ** -3),
                            (dX - dY, x.grad - ref.d(dY), 2.0 ** -4 + 2.0 ** -3)):
        have, want = ref.d(have), ref.d(want)
        # (Y − X and dX − dY hold the rounding of the stored sums too)
        slack = 2.0 ** -8 * float(torch.cat((ref.d(Y).flatten(), ref.d(dX).flatten())).norm())
        assert float((have - want).norm()) <= off * float(want.norm()) + slack


def test_same_bits_on_another_stream_and_in_a_graph(L):
    gen = torch.Generator().manual_seed(9)
    M, D = 200, 384
    X, dY = rows(gen, M, D, BF16).cuda(), torch.randn(M, D, generator=gen).to(BF16).cuda()
    w, b = torch.randn(D, generator=gen).cuda(), torch.randn(D, generator=gen).cuda()
    W = (torch.randn(D, D, generator=gen) * D ** -0.5).to(BF16).cuda()
    want = block(L, X, w, b, W, dY)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = block(L, X, w, b, W, dY)
    s.synchronize()
    for a, c in zip(got, want):
        assert torch.equal(a, c)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = block(L, X, w, b, W, dY)
    for k in range(4):
        X.copy_(rows(torch.Generator().manual_seed(20 + k), M, D, BF16))
        dY.mul_(-0.5)
        for t in held:
            t.fill_(math.nan)
        g.replay()
        torch.cuda.synchronize()
        for a, c in zip(held, block(L, X, w, b, W, dY)):
            assert torch.equal(a, c)


def test_streams_given_by_handle(L):
    """Calls on a stream given as an argument: outputs allocated for it."""
    gen = torch.Generator().manual_seed(2)
    X = rows(gen, 70, 200).cuda()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    q = L.gt_quantise(X, need=("codes", "transposed"), stream=s)
    n = L.gt_norm_fp8(X, stream=s.cuda_stream)
    y = L.gt_linear_fp8(n, q.codes, stream=s)
    s.synchronize()
    want = L.gt_linear_fp8(L.gt_norm_fp8(X), L.gt_quantise(X).codes)
    torch.cuda.synchronize()
    assert torch.equal(y, want)
