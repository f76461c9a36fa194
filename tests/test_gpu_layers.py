"""The layer operators on the GPU against their definitions in 64 bits
(layers_plain), every value within its own rounding bound; what lies around
the operands is NaN and must not be read into a result, what lies around the
outputs must stay as it was."""
import itertools
import math

import pytest
import torch

import layers_plain as ref

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
IDS = {BF16: "bf16", F32: "f32"}


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_1909_10616_amd import layers
    layers.lib()
    return layers


def note(msg):
    print(msg, flush=True)


class Frame:
    """Operands laid inside larger NaN-filled buffers, outputs inside buffers whose
    surroundings are checked afterwards."""

    def __init__(self, seed, pad):
        self.gen = torch.Generator().manual_seed(seed)
        self.pad, self.outputs = pad, []

    def normal(self, dtype, *shape, std=1.0):
        return self.place((torch.randn(*shape, generator=self.gen) * std).to(dtype))

    def ints(self, dtype, *shape, most=3):
        return self.place(torch.randint(-most, most + 1, shape, generator=self.gen).to(dtype))

    def place(self, t):
        if not self.pad or t.dim() < 2:
            return t.cuda()
        buf = torch.full((*t.shape[:-2], t.shape[-2] + 3, t.shape[-1] + self.pad), float("nan"),
                         dtype=t.dtype, device="cuda")
        view = buf[..., 1:1 + t.shape[-2], :t.shape[-1]]
        view.copy_(t)
        return view

    def output(self, dtype, *shape):
        buf = torch.full((shape[0] + 3, shape[1] + self.pad), -77.0, dtype=dtype, device="cuda")
        view = buf[1:1 + shape[0], :shape[1]]
        self.outputs.append((buf, shape))
        return view

    def untouched(self):
        for buf, (m, n) in self.outputs:
            rest = torch.ones_like(buf, dtype=torch.bool)
            rest[1:1 + m, :n] = False
            assert bool((buf[rest] == -77.0).all())


# ---------------------------------------------------------------------------
# linear
# ---------------------------------------------------------------------------

SHAPES = [(1, 1, 1), (1, 64, 64), (1, 133, 1), (1, 1024, 520), (3, 130, 77), (16, 128, 64),
          (17, 136, 200), (64, 64, 64), (65, 72, 24), (130, 131, 129), (129, 257, 65), (250, 264, 512),
          (257, 512, 40), (300, 520, 1032)]


@pytest.mark.parametrize("pad", [0, 8, 5])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dtype", [BF16, F32], ids=IDS.get)
def test_linear(L, dtype, shape, pad):
    M, N, K = shape
    for i, (act, gated) in enumerate(itertools.product(("none", "relu", "gelu", "silu"), (False, True))):
        f = Frame(i, pad)
        wide = N * (2 if gated else 1)
        note(f"linear {dtype} {shape} pad {pad} {act} gated {gated}")
        X, W = f.normal(dtype, M, K), f.normal(dtype, K, wide, std=K ** -0.5)
        bias = f.normal(dtype, wide) if i % 3 else None
        R = f.normal(dtype, M, N) if i % 2 else None
        P = f.output(dtype, M, wide) if i % 4 != 1 else None
        Y = f.output(F32 if i == 2 else dtype, M, N)
        assert L.gt_linear(X, W, bias=bias, residual=R, act=act, gated=gated, Y=Y, P=P) is Y
        torch.cuda.synchronize()
        want, pre = ref.linear(X, W, bias, R, act, gated, out=Y.dtype)
        ref.check(Y, want, "Y")
        if P is not None:
            ref.check(P, pre, "P")
        f.untouched()


# every tile, K long enough for K slices, and rows past the largest tile
LARGE = [(BF16, 520, 768, 320), (BF16, 1, 264, 8200), (BF16, 12, 520, 8192), (BF16, 64, 256, 8200),
         (BF16, 1030, 1032, 200), (BF16, 515, 1021, 333), (F32, 12, 264, 4100), (F32, 260, 516, 260),
         (F32, 333, 255, 1027), (BF16, 2050, 2056, 136)]


@pytest.mark.parametrize("case", LARGE, ids=lambda c: f"{IDS[c[0]]}-{c[1]}x{c[2]}x{c[3]}")
def test_linear_whole_numbers(L, case):
    """Products of small whole numbers are exact in fp32, in any order and on any path."""
    dtype, M, N, K = case
    f = Frame(5, 0)
    note(f"linear exact {case}")
    X, W, R = f.ints(dtype, M, K), f.ints(dtype, K, N), f.ints(dtype, M, N)
    Y = f.output(F32, M, N)
    L.gt_linear(X, W, residual=R, Y=Y)
    want = (X.float().cpu() @ W.float().cpu() + R.float().cpu())
    assert torch.equal(Y.cpu(), want)
    f.untouched()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=IDS.get)
def test_linear_same_bits_and_residual_in_place(L, dtype):
    f = Frame(7, 0)
    X, W, R = f.normal(dtype, 33, 4096), f.normal(dtype, 4096, 264), f.normal(dtype, 33, 264)
    first = L.gt_linear(X, W, residual=R, act="gelu")
    for _ in range(3):
        assert torch.equal(L.gt_linear(X, W, residual=R, act="gelu"), first)
    Y = R.clone()
    L.gt_linear(X, W, residual=Y, act="gelu", Y=Y)
    assert torch.equal(Y, first)


def test_linear_no_rows(L):
    X, W = torch.zeros(0, 16, device="cuda"), torch.randn(16, 24, device="cuda")
    assert L.gt_linear(X, W).shape == (0, 24)
    dX, dW, db = L.gt_linear_backward(torch.zeros(0, 24, device="cuda"), X, W, act="none")
    assert dX.shape == (0, 16) and not dW.any() and not db.any() and dW.shape == W.shape


def test_linear_infinities_and_nan_stay_in_their_rows(L):
    f = Frame(3, 0)
    X, W = f.normal(BF16, 70, 96), f.normal(BF16, 96, 136)
    clean = L.gt_linear(X, W, act="relu")
    X[5, 7], X[40, 3] = math.nan, math.inf
    Y = L.gt_linear(X, W, act="relu")
    assert bool(Y[5].isnan().all())
    assert bool((Y[40].isinf() | (Y[40] == 0)).all()) and bool(Y[40].isinf().any())
    rest = [r for r in range(70) if r not in (5, 40)]
    assert torch.equal(Y[rest], clean[rest])


def test_linear_far_offsets(L):
    """Rows more than 2^31 elements into their array."""
    ld = 1 << 20
    big = torch.empty(2304 * ld, dtype=BF16, device="cuda")
    X = big.view(2304, ld)[:, :64]
    g = torch.Generator().manual_seed(1)
    X.copy_(torch.randint(-3, 4, (2304, 64), generator=g).to(BF16))
    W = torch.randint(-3, 4, (64, 72), generator=g).to(BF16).cuda()
    Y = L.gt_linear(X, W, Y=torch.empty(2304, 72, device="cuda"))
    assert torch.equal(Y.cpu(), X.float().cpu() @ W.float().cpu())
    out = big.view(2304, ld)[:, 128:200]
    L.gt_linear(X, W, Y=out)
    assert torch.equal(out.float().cpu(), Y.bfloat16().float().cpu())


# ---------------------------------------------------------------------------
# linear's gradients
# ---------------------------------------------------------------------------

GRAD_SHAPES = [(1, 1, 1), (1, 72, 130), (5, 64, 8), (64, 64, 64), (66, 131, 77), (129, 136, 264),
               (513, 40, 24), (200, 520, 300), (1030, 72, 65)]


@pytest.mark.parametrize("pad", [0, 5])
@pytest.mark.parametrize("shape", GRAD_SHAPES, ids=str)
@pytest.mark.parametrize("dtype", [BF16, F32], ids=IDS.get)
def test_linear_backward(L, dtype, shape, pad):
    M, N, K = shape
    for i, (act, gated) in enumerate(itertools.product(("none", "relu", "gelu", "silu"), (False, True))):
        f = Frame(i, pad)
        wide = N * (2 if gated else 1)
        note(f"linear_backward {dtype} {shape} pad {pad} {act} gated {gated}")
        X, W, dY = f.normal(dtype, M, K), f.normal(dtype, K, wide), f.normal(dtype, M, N)
        P = f.normal(dtype, M, wide)
        out = F32 if i == 5 else dtype
        dX, dW = f.output(dtype, M, K), f.output(out, K, wide)
        got = L.gt_linear_backward(dY, X, W, P=P, act=act, gated=gated, dX=dX, dW=dW)
        torch.cuda.synchronize()
        want = ref.linear_backward(dY, X, W, P, act, gated, dtype, out)
        for name, g, w in zip(("dX", "dW", "db"), got, want):
            ref.check(g, w, name)
        f.untouched()


def test_linear_backward_wanted_parts(L):
    f = Frame(1, 0)
    X, W, P, dY = f.normal(F32, 40, 24), f.normal(F32, 24, 32), f.normal(F32, 40, 32), f.normal(F32, 40, 32)
    dX, dW, db = L.gt_linear_backward(dY, X, W, P=P, act="silu")
    assert torch.equal(L.gt_linear_backward(dY, X, W, P=P, act="silu", need=("dX",), bias=False)[0], dX)
    got = L.gt_linear_backward(dY, X, W, P=P, act="silu", need=("dW",), bias=False)
    assert got[0] is None and got[2] is None and torch.equal(got[1], dW)
    got = L.gt_linear_backward(dY, X, W, P=P, act="silu", need=())
    assert got[0] is None and got[1] is None and torch.equal(got[2], db)


@pytest.mark.parametrize("act,gated", [("gelu", False), ("silu", True), ("none", True)])
def test_linear_gradients_against_differences(L, act, gated):
    """(Y(p + h) − Y(p − h)) / 2h along a direction, from fp32 outputs: the step's third-order
    term and the rounding of Y are far below the 1e-3 the comparison allows."""
    f = Frame(2, 0)
    M, N, K = 9, 12, 10
    wide = N * (2 if gated else 1)
    X, W, b = f.normal(F32, M, K), f.normal(F32, K, wide, std=0.5), f.normal(F32, wide)
    dY = f.normal(F32, M, N)
    P = torch.empty(M, wide, device="cuda")
    L.gt_linear(X, W, bias=b, act=act, gated=gated, P=P)
    grads = L.gt_linear_backward(dY, X, W, P=P, act=act, gated=gated)
    h = 2.0 ** -7
    for i, g in enumerate(grads):
        args = [X, W, b]
        dir_ = f.normal(F32, *args[i].shape)
        val = []
        for sign in (1, -1):
            a = list(args)
            a[i] = args[i] + sign * h * dir_
            Y = L.gt_linear(a[0], a[1], bias=a[2], act=act, gated=gated)
            val.append((Y.double() * dY.double()).sum().item())
        want = (val[0] - val[1]) / (2 * h)
        have = (g.double() * dir_.double()).sum().item()
        scale = (g.double().abs() * dir_.double().abs()).sum().item()
        assert abs(have - want) <= 1e-3 * scale


# ---------------------------------------------------------------------------
# routing
# ---------------------------------------------------------------------------

ROUTES = [
    # T, E, k, score, groups, keep, bias, renormalise
    (1, 1, 1, "softmax", 1, 1, False, True), (1, 8, 2, "softmax", 1, 1, False, False),
    (5, 7, 7, "sigmoid", 1, 1, True, True), (64, 64, 6, "softmax", 1, 1, True, True),
    (33, 60, 4, "sigmoid", 4, 2, True, False), (65, 128, 8, "softmax", 8, 3, False, True),
    (300, 256, 8, "sigmoid", 8, 4, True, True), (130, 257, 3, "softmax", 1, 1, True, False),
    (70, 512, 16, "softmax", 64, 10, False, True), (9, 1000, 20, "sigmoid", 10, 5, True, True),
    (700, 16, 2, "softmax", 16, 3, True, True), (2, 1024, 64, "softmax", 1024, 64, False, False),
    (40, 96, 64, "sigmoid", 1, 1, False, True),
]


def logits_for(kind, T, E, gen):
    x = torch.randn(T, E, generator=gen) * 2
    if kind == "ties":
        x = (x * 2).round() / 2
    elif kind == "holes":     # shut experts, whole rows without any, NaN and infinities
        x[torch.rand(T, E, generator=gen) < 0.3] = -math.inf
        x[torch.rand(T, generator=gen) < 0.2] = -math.inf
        x[torch.rand(T, E, generator=gen) < 0.02] = math.nan
        x[torch.rand(T, E, generator=gen) < 0.01] = math.inf
        x[torch.rand(T, E, generator=gen) < 0.02] = torch.finfo(BF16).min
    elif kind == "far":       # scores too small for a float
        x = x * 100
    return x


@pytest.mark.parametrize("kind", ["plain", "ties", "holes", "far"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS.get)
@pytest.mark.parametrize("case", ROUTES, ids=str)
def test_route(L, case, dtype, kind):
    T, E, k, score, groups, keep, bias, renorm = case
    gen = torch.Generator().manual_seed(T * E + k)
    note(f"route {case} {dtype} {kind}")
    x = logits_for(kind, T, E, gen).to(dtype)
    buf = torch.full((T + 1, E + 3), math.nan, dtype=dtype, device="cuda")
    logits = buf[:T, :E]
    logits.copy_(x)
    b = (torch.randint(-8, 9, (E,), generator=gen) / 8.0) if bias else None
    scale = 2.5
    r = L.gt_route(logits, k, bias=None if b is None else b.cuda(), score=score, groups=groups,
                   keep=keep, renormalise=renorm, scale=scale)
    want = ref.choose(x, k, b, groups, keep)
    assert torch.equal(r.experts.cpu().long(), want)
    for got, w in zip((r.offsets, r.order, r.place), ref.lists(want, E)):
        assert torch.equal(got.cpu(), w)
    # a share: the exponential of a difference rounded at |x|·2^-24 (absolute error of the
    # exponent), sums of E terms, quotients
    part, sc = ref.shares(x, want, score, renorm)
    far = float(x.double().nan_to_num(0, 0, 0).abs().clamp(max=1e4).max())
    rel = (E + 32 + 2 * far) * ref.EPS
    ref.check(r.weights, (scale * part, scale * part * rel + 1e-37), "weights")

    dw = torch.randn(T, k, generator=gen)
    out = torch.full((T + 1, E + 3), -77.0, dtype=dtype, device="cuda")
    g = L.gt_route_backward(dw.cuda(), logits, r.experts, score=score, renormalise=renorm, scale=scale,
                            dlogits=out[:T, :E])
    value, size = ref.route_backward(x, want, dw, score, renorm, scale)
    assert bool((out[T] == -77.0).all()) and bool((out[:, E:] == -77.0).all())
    ref.check(g, ref.stored(value, size * 4 * rel + 1e-37, dtype), "dlogits")


def test_route_no_tokens(L):
    r = L.gt_route(torch.zeros(0, 8, device="cuda"), 2)
    assert r.weights.shape == (0, 2) and not r.offsets.any() and r.order.numel() == 0
    assert L.gt_route_backward(r.weights, torch.zeros(0, 8, device="cuda"), r.experts).shape == (0, 8)


def test_route_many_blocks(L):
    """More entries than one sort block per expert, all going to few experts."""
    gen = torch.Generator().manual_seed(0)
    x = torch.randn(5000, 32, generator=gen).round()
    x[:, 20:] -= 100
    r = L.gt_route(x.cuda(), 4)
    want = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :4]
    assert torch.equal(r.experts.cpu().long(), want)
    for got, w in zip((r.offsets, r.order, r.place), ref.lists(want, 32)):
        assert torch.equal(got.cpu(), w)


# ---------------------------------------------------------------------------
# experts
# ---------------------------------------------------------------------------

EXPERTS = [
    # T, E, k, D, H
    (1, 1, 1, 8, 8), (1, 8, 2, 64, 72), (3, 5, 3, 33, 17), (40, 4, 2, 136, 64), (70, 3, 1, 64, 200),
    (150, 6, 2, 264, 130), (300, 2, 2, 72, 136), (64, 40, 4, 128, 64), (20, 70, 1, 24, 40),
]


def routed(L, f, T, E, k, holes):
    x = torch.randn(T, E, generator=f.gen) * 2
    if holes:
        x[:, 0] = -math.inf                                  # an expert without rows
        x[torch.rand(T, generator=f.gen) < 0.3] = -math.inf  # tokens without experts
    return L.gt_route(x.cuda(), k, renormalise=False, scale=1.5)


@pytest.mark.parametrize("holes", [False, True])
@pytest.mark.parametrize("pad", [0, 8, 3])
@pytest.mark.parametrize("case", EXPERTS, ids=str)
@pytest.mark.parametrize("dtype", [BF16, F32], ids=IDS.get)
def test_experts_and_their_gradients(L, dtype, case, pad, holes):
    T, E, k, D, H = case
    for i, (act, gated) in enumerate((("silu", True), ("gelu", False), ("relu", True), ("none", False))):
        f = Frame(10 * i + T, pad)
        note(f"experts {dtype} {case} pad {pad} holes {holes} {act} gated {gated}")
        r = routed(L, f, T, E, k, holes)
        wide = H * (2 if gated else 1)
        X = f.normal(dtype, T, D)
        W1, W2 = f.normal(dtype, E, D, wide, std=D ** -0.5), f.normal(dtype, E, H, D, std=H ** -0.5)
        b1 = f.normal(dtype, E, wide).contiguous() if i != 2 else None
        b2 = f.normal(dtype, E, D).contiguous() if i != 2 else None
        R = f.normal(dtype, T, D) if i % 2 == 0 else None
        Y, P = f.output(dtype, T, D), f.output(dtype, T * k, wide)
        L.gt_experts(X, r, W1, W2, b1=b1, b2=b2, residual=R, act=act, gated=gated, Y=Y, P=P)
        chosen, order = r.experts.cpu().long(), r.order.cpu()
        want, pre = ref.experts(X, W1, W2, r.weights, chosen, order, b1, b2, R, act, gated, dtype)
        ref.check(Y, want, "Y")
        n = pre[0].shape[0]
        ref.check(P[:n], pre, "P")
        assert bool((P[n:] == -77.0).all())
        f.untouched()

        dY = f.normal(dtype, T, D)
        Pn = P.clone()
        Pn[n:] = math.nan
        got = L.gt_experts_backward(dY, X, r, W1, W2, Pn, b2=b2, act=act, gated=gated)
        grads = ref.experts_backward(dY, X, W1, W2, Pn[:n], r.weights, chosen, order, b2, act, gated, dtype)
        for name, w in grads.items():
            ref.check(getattr(got, name), w, name)


@pytest.mark.parametrize("dtype,T,E,k,D,H", [(BF16, 600, 3, 2, 256, 264), (BF16, 1100, 2, 1, 520, 128),
                                             (F32, 400, 3, 1, 132, 260)])
def test_experts_whole_numbers(L, dtype, T, E, k, D, H):
    """Large enough for the largest tiles; small whole numbers, exact throughout: weights a power
    of two, activations below 2^8 in bf16."""
    f = Frame(4, 0)
    note(f"experts exact {dtype} {T} {E} {k} {D} {H}")
    r = routed(L, f, T, E, k, False)
    r = r._replace(weights=torch.full_like(r.weights, 0.5))
    X = torch.zeros(T, D, dtype=dtype)
    X[torch.arange(T), torch.randint(0, D, (T,), generator=f.gen)] = 2.0
    W1, W2 = f.ints(dtype, E, D, H), f.ints(dtype, E, H, D, most=1)
    Xd = X.cuda()
    Y = L.gt_experts(Xd, r, W1, W2, act="relu", Y=None)
    want = torch.zeros(T, D, dtype=torch.float64)
    chosen = r.experts.cpu().long()
    for t in range(T):
        for s in range(k):
            e = int(chosen[t, s])
            h = (X[t].double() @ W1[e].cpu().double()).clamp(min=0)
            want[t] += 0.5 * (h @ W2[e].cpu().double())
    assert torch.equal(Y.cpu(), want.to(dtype))


def test_experts_no_tokens(L):
    r = L.gt_route(torch.zeros(0, 4, device="cuda"), 2)
    X = torch.zeros(0, 16, dtype=BF16, device="cuda")
    W1, W2 = torch.ones(4, 16, 24, dtype=BF16, device="cuda"), torch.ones(4, 24, 16, dtype=BF16, device="cuda")
    assert L.gt_experts(X, r, W1, W2).shape == (0, 16)
    g = L.gt_experts_backward(X, X, r, W1, W2, torch.zeros(0, 24, dtype=BF16, device="cuda"))
    assert not g.dW1.any() and not g.dW2.any() and not g.db1.any() and not g.db2.any()
    assert g.dX.shape == (0, 16) and g.dweights.shape == (0, 2)


def test_lists_out_of_range_are_no_expert(L):
    """Entries of `place` and `order` outside their range take no part."""
    f = Frame(6, 0)
    r = routed(L, f, 20, 4, 2, False)
    X = f.normal(BF16, 20, 64)
    W1, W2 = f.normal(BF16, 4, 64, 72), f.normal(BF16, 4, 72, 64)
    place = r.place.clone()
    place[3], place[7, 1] = 1 << 30, -5
    Y = L.gt_experts(X, r._replace(place=place), W1, W2)
    weights = r.weights.clone()
    weights[3], weights[7, 1] = 0, 0
    assert torch.equal(Y, L.gt_experts(X, r._replace(weights=weights), W1, W2))


# ---------------------------------------------------------------------------
# streams, graphs, workspaces
# ---------------------------------------------------------------------------

def test_other_stream_and_given_workspace(L):
    f = Frame(8, 0)
    X, W = f.normal(BF16, 16, 8192), f.normal(BF16, 8192, 256)
    want = L.gt_linear(X, W, act="silu")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = L.gt_linear(X, W, act="silu", stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    ws = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")
    assert torch.equal(L.gt_linear(X, W, act="silu", workspace=ws), want)
    from paper_1909_10616_amd.gemmtune import GemmTuneError
    with pytest.raises(GemmTuneError, match="workspace"):
        L.gt_linear(X, W, act="silu", workspace=ws[:256])


def test_whole_layer_in_a_graph(L):
    """Router product, routing, experts and all gradients captured once and replayed on
    new inputs, each replay equal to the eager calls."""
    f = Frame(9, 0)
    T, E, k, D, H = 96, 8, 2, 64, 128
    X, dY = f.normal(BF16, T, D), f.normal(BF16, T, D)
    Wr = f.normal(BF16, D, E)
    W1, W2 = f.normal(BF16, E, D, 2 * H, std=0.1), f.normal(BF16, E, H, D, std=0.1)
    P = torch.empty(T * k, 2 * H, dtype=BF16, device="cuda")

    def step():
        logits = L.gt_linear(X, Wr)
        r = L.gt_route(logits, k)
        Y = L.gt_experts(X, r, W1, W2, residual=X, gated=True, P=P)
        g = L.gt_experts_backward(dY, X, r, W1, W2, P, gated=True, bias=False)
        dl = L.gt_route_backward(g.dweights, logits, r.experts)
        dx, dwr, _ = L.gt_linear_backward(dl, X, Wr, bias=False)
        return [Y, g.dX, g.dW1, g.dW2, dl, dx, dwr]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for n in range(4):
        X.copy_(f.normal(BF16, T, D))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        for a, b in zip(got, step()):
            assert torch.equal(a, b)
        torch.cuda.synchronize()
