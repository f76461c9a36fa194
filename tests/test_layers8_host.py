"""The norm's, the quantising's and the 8-bit layers' entry points without a GPU: wrong
arguments are refused before anything is launched, the scratch queries survive
arbitrary argument values, the last sizes that are served, and what the binding refuses."""
import ctypes
import random

import pytest
import torch

from test_layers_host import AT, GT_EINVAL, GT_ESMALL, VALUES, message

M, N, K = 5, 260, 300
VALID = {
    "gt_quantise": dict(M=M, N=N, dtype=1, code=0, block=1, pow2=0, X=AT, ldx=N, Q=AT, ldq=N, S=AT, lds=3, Qt=AT,
                        ldqt=M, St=AT, ldst=1),
    "gt_linear_fp8": dict(M=M, N=N, K=K, dtype=1, act=19, out_dtype=1, xcode=0, wcode=1, xblock=1, wblock=128, X=AT,
                          ldx=304, sx=AT, ldsx=3, W=AT, ldw=304, sw=AT, ldsw=3, bias=AT, R=AT, ldr=N, Y=AT + 4096,
                          ldy=N),
    "gt_norm": dict(M=M, N=N, dtype=1, wtype=0, code=0, pow2=1, eps=1e-5, X=AT, ldx=N, w=AT, b=AT, Y=AT + 65536,
                    ldy=N, mean=AT, rstd=AT, Q=AT, ldq=N, S=AT, lds=3),
    "gt_norm_backward": dict(M=M, N=N, dtype=1, wtype=1, dY=AT, lddy=N, X=AT, ldx=N, w=AT, mean=AT, rstd=AT, R=AT,
                             ldr=N, dX=AT + 65536, lddx=N, dw=AT, db=AT),
}
WRONG = {
    "gt_quantise": [dict(M=-1), dict(N=0), dict(M=1 << 31), dict(N=1 << 31), dict(dtype=2), dict(code=2),
                    dict(code=-1), dict(block=0), dict(block=64), dict(X=None), dict(Q=None, Qt=None), dict(S=None),
                    dict(St=None), dict(ldx=N - 1), dict(ldq=N - 1), dict(lds=2), dict(ldqt=M - 1), dict(ldst=0),
                    dict(X=AT + 1), dict(S=AT + 2), dict(St=AT + 1), dict(ldx=1 << 31),
                    dict(M=(1 << 31) - 1, ldx=1 << 20)],
    "gt_linear_fp8": [dict(M=-1), dict(N=0), dict(K=0), dict(N=1 << 30), dict(dtype=2), dict(act=4), dict(act=32),
                      dict(out_dtype=2), dict(dtype=0, out_dtype=1), dict(xcode=2), dict(wcode=-1), dict(xblock=2),
                      dict(wblock=0), dict(X=None), dict(sx=None), dict(W=None), dict(sw=None), dict(Y=None),
                      dict(ldx=K - 1), dict(ldw=K - 1), dict(ldsx=2), dict(ldsw=2), dict(ldr=N - 1), dict(ldy=N - 1),
                      dict(sx=AT + 2), dict(sw=AT + 1), dict(bias=AT + 1), dict(R=AT + 1), dict(Y=AT + 1),
                      dict(out_dtype=0, R=AT, Y=AT), dict(R=AT, Y=AT, ldr=N + 1), dict(ldx=1 << 31),
                      dict(M=(1 << 31) - 1, ldx=1 << 20)],
    "gt_norm": [dict(M=-1), dict(N=0), dict(dtype=2), dict(wtype=2), dict(dtype=0, wtype=1), dict(code=2),
                dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(X=None),
                dict(Y=None, Q=None, mean=None, rstd=None), dict(S=None), dict(ldx=N - 1), dict(ldy=N - 1),
                dict(ldq=N - 1), dict(lds=2), dict(X=AT + 1), dict(w=AT + 2), dict(b=AT + 1), dict(Y=AT + 1),
                dict(mean=AT + 2), dict(rstd=AT + 1), dict(S=AT + 1), dict(Y=AT, ldy=N + 8), dict(ldx=1 << 31)],
    "gt_norm_backward": [dict(M=-1), dict(N=0), dict(dtype=3), dict(wtype=-1), dict(dtype=0, wtype=1), dict(dY=None),
                         dict(X=None), dict(mean=None), dict(rstd=None), dict(lddy=N - 1), dict(ldx=N - 1),
                         dict(ldr=N - 1), dict(lddx=N - 1), dict(dY=AT + 1), dict(w=AT + 1), dict(mean=AT + 2),
                         dict(dX=AT + 1), dict(dw=AT + 2), dict(db=AT + 1), dict(dX=AT, lddx=N + 1),
                         dict(dX=AT, R=None, lddx=N + 8)],
}


@pytest.fixture(scope="module")
def L():
    from paper_1909_10616_amd import layers
    layers.lib()
    return layers


def args(L, name, **change):
    a = L.EXPORTS[name]()
    for f, v in {**VALID[name], **change}.items():
        setattr(a, f, v)
    return a


def call(L, name, a, ws=AT, ws_bytes=1 << 40):
    f = getattr(L.lib(), name)
    return f(ctypes.byref(a), None) if name in L.NO_SCRATCH else f(ctypes.byref(a), ws, ws_bytes, None)


@pytest.mark.parametrize("name,change", [(n, c) for n, cs in WRONG.items() for c in cs],
                         ids=lambda v: v if isinstance(v, str) else ",".join(f"{k}={x}" for k, x in v.items()))
def test_wrong_arguments_are_refused(L, name, change):
    assert call(L, name, args(L, name, **change)) == GT_EINVAL
    assert message(L)


@pytest.mark.parametrize("name", VALID)
def test_null_arguments_are_refused(L, name):
    f = getattr(L.lib(), name)
    assert (f(None, None) if name in L.NO_SCRATCH else f(None, AT, 1 << 40, None)) == GT_EINVAL
    if name not in L.NO_SCRATCH:
        w = getattr(L.lib(), name + "_workspace")
        n = ctypes.c_int64()
        assert w(None, ctypes.byref(n)) == GT_EINVAL
        assert w(ctypes.byref(args(L, name)), None) == GT_EINVAL


# K slices; rows at odd addresses, copied; the column sums
@pytest.mark.parametrize("name,change", [
    ("gt_linear_fp8", dict(M=256, N=2048, K=8192, ldx=8192, ldw=8192, ldsx=64, ldsw=64, act=0, ldr=2048, ldy=2048)),
    ("gt_linear_fp8", dict(M=3000, N=2048, K=4099, ldx=4099, ldw=4099, ldsx=33, ldsw=33, act=0, ldr=2048, ldy=2048)),
    ("gt_norm_backward", dict(M=1025))])
def test_scratch_too_small_or_misaligned(L, name, change):
    a = args(L, name, **change)
    need = L.workspace_bytes(name, a)
    assert need > 0
    assert call(L, name, a, AT, need - 1) == GT_ESMALL and str(need) in message(L)
    assert call(L, name, a, AT, 0) == GT_ESMALL
    assert call(L, name, a, None, need) == GT_EINVAL
    assert call(L, name, a, AT + 16, need) == GT_EINVAL


def test_sums_of_few_rows_need_no_scratch(L):
    """Whatever is wanted and wherever dX lies."""
    for change in ({}, dict(dX=AT), dict(dX=None), dict(dw=None), dict(M=1024), dict(N=16384)):
        n = dict(N=16384, lddy=16384, ldx=16384, ldr=16384, lddx=16384) if "N" in change else {}
        assert L.workspace_bytes("gt_norm_backward", args(L, "gt_norm_backward", **{**change, **n})) == 0
    assert L.workspace_bytes("gt_norm_backward", args(L, "gt_norm_backward", M=1025)) > 0


def test_copies_are_as_large_as_the_rows(L):
    """Both operands at odd addresses: their rows of whole 16-byte chunks, side by side."""
    a = args(L, "gt_linear_fp8", M=3000, N=2048, K=4099, ldx=4099, ldw=4099, ldsx=33, ldsw=33, act=0, ldr=2048,
             ldy=2048)
    up = lambda v, m: -(-v // m) * m  # noqa: E731
    assert L.workspace_bytes("gt_linear_fp8", a) >= up(3000 * 4112, 256) + up(2048 * 4112, 256)
    b = args(L, "gt_linear_fp8", M=3000, N=2048, K=4099, ldx=4112, ldw=4112, ldsx=33, ldsw=33, act=0, ldr=2048,
             ldy=2048)
    assert L.workspace_bytes("gt_linear_fp8", b) == 0


def test_no_rows_need_nothing(L):
    for name in VALID:
        a = args(L, name, M=0)
        if name not in L.NO_SCRATCH:
            assert L.workspace_bytes(name, a) == 0
        if name != "gt_norm_backward":   # (its sums of no rows are written)
            assert call(L, name, args(L, name, M=0, X=None), None, 0) == 0
    a = args(L, "gt_norm_backward", M=0, dY=None, X=None, mean=None, rstd=None, dw=None, db=None)
    assert call(L, "gt_norm_backward", a, None, 0) == 0


@pytest.mark.parametrize("name", [n for n in VALID if n not in ("gt_quantise", "gt_norm")])
def test_queries_survive_arbitrary_arguments(L, name):
    rng = random.Random(name)
    served = 0
    for i in range(4000):
        a = args(L, name)
        for f, t in a._fields_:
            if rng.random() >= (0.12 if i % 2 else 0.5):
                continue
            if t is ctypes.c_void_p:
                setattr(a, f, rng.choice([None, AT, AT + 1, AT + 2, AT + 4, AT + 16]))
            elif t is ctypes.c_float:
                setattr(a, f, rng.choice([0.0, float("nan"), 1e30]))
            else:
                v = rng.choice(VALUES)
                setattr(a, f, v if ctypes.sizeof(t) == 8 else max(-(1 << 31), min(v, (1 << 31) - 1)))
        n = ctypes.c_int64(-1)
        rc = getattr(L.lib(), name + "_workspace")(ctypes.byref(a), ctypes.byref(n))
        assert rc in (0, GT_EINVAL)
        if rc == 0:
            served += 1
            assert 0 <= n.value < 1 << 62
        else:
            assert n.value == -1 and message(L)
    assert served > 20


def test_every_size_has_a_form(L):
    """From one row to the largest, aligned or not, an answer within the scratch that a GPU has."""
    for m in (1, 2, 16, 17, 33, 64, 65, 100, 999, 4096, 65536, 302 << 20):
        for n in (1, 7, 64, 1021, 4096, 11008):
            for k in (1, 127, 128, 777, 4096, 65536):
                for act in (0, 19):
                    for pad in (0, 1):
                        if m * max(n, k) > 1 << 36:
                            continue
                        ld = (k + 15) // 16 * 16 + pad
                        kb = -(-k // 128)
                        a = args(L, "gt_linear_fp8", M=m, N=n, K=k, act=act, ldx=ld, ldw=ld, ldsx=kb, ldsw=kb, ldr=n,
                                 ldy=n)
                        need = L.workspace_bytes("gt_linear_fp8", a)
                        assert 0 <= need <= 2 * (m + 2 * n) * (ld + 16) + 16 * m * 2 * (n + 4) * 4 + 4096


def test_more_rows_than_any_form_takes(L):
    a = args(L, "gt_linear_fp8", M=(1 << 31) - 1, N=300, K=1, act=0, ldx=16, ldw=16, ldsx=1, ldsw=1, ldr=300, ldy=300)
    assert call(L, "gt_linear_fp8", a) == GT_EINVAL and "too many rows" in message(L)


def test_wide_norms_need_few_partial_sums(L):
    for n in (1, 1000, 8192, 8193, 16385, 1 << 20):
        a = args(L, "gt_norm_backward", M=1 << 20, N=n, lddy=n, ldx=n, ldr=n, lddx=n)
        assert L.workspace_bytes("gt_norm_backward", a) <= 512 * 8 * n + 256
        a = args(L, "gt_norm_backward", M=1 << 20, N=n, lddy=n, ldx=n, ldr=n, lddx=n, dw=None, db=None)
        assert L.workspace_bytes("gt_norm_backward", a) == 0


# ---------------------------------------------------------------------------
# the Python side
# ---------------------------------------------------------------------------

def test_cpu_tensors_are_refused(L):
    X, s = torch.zeros(4, 128), torch.zeros(4, 1)
    q = L.Codes(torch.zeros(4, 128, dtype=torch.uint8).view(torch.float8_e4m3fn), s)
    v = torch.zeros(4)
    for f in (lambda: L.gt_norm(X), lambda: L.gt_norm_fp8(X), lambda: L.gt_norm_backward(X, X, v, v),
              lambda: L.gt_quantise(X), lambda: L.gt_linear_fp8(q, q)):
        with pytest.raises(ValueError, match="GPU tensor"):
            f()


def test_codes_are_asked_for(L):
    X = torch.zeros(4, 128)
    for x, w in ((X, X), (None, None), (L.Codes(X, X), 3), (3, L.Codes(X, X)), ((), ()), ((3, 4), L.Codes(X, X)),
                 (L.Codes(X, X), X)):
        with pytest.raises(ValueError):
            L.gt_linear_fp8(x, w)
