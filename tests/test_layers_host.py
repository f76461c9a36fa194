"""The layer operators' entry points without a GPU: the binding agrees with the
header, wrong arguments are refused before anything is launched, and the
scratch queries survive arbitrary argument values."""
import ctypes
import os
import random
import re
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "gemmtune_layers.h")
GT_EINVAL, GT_ESMALL = -1, -7
AT = 1 << 20      # an aligned address nothing reads


@pytest.fixture(scope="module")
def L():
    from paper_1909_10616_amd import layers
    layers.lib()
    return layers


def test_status_codes():
    text = open(os.path.join(ROOT, "include", "gemmtune.h")).read()
    assert re.search(r"GT_EINVAL\s*=\s*%d\b" % GT_EINVAL, text)
    assert re.search(r"GT_ESMALL\s*=\s*%d\b" % GT_ESMALL, text)


def test_header_symbols_are_exported_and_bound(L):
    names = set(re.findall(r"^int (gt_\w+)\(", open(HEADER).read(), re.M))
    bound = set(L.EXPORTS) | {n + "_workspace" for n in L.EXPORTS if n not in L.NO_SCRATCH}
    assert names == bound
    for n in names:
        assert getattr(L.lib(), n)


def test_structures_are_the_headers(L, tmp_path):
    """Size and every field's offset, from a C compiler."""
    lines = []
    for t in L.EXPORTS.values():
        lines.append(f'printf("{t.__name__} %zu\\n", sizeof({t.__name__}));')
        lines += [f'printf("{t.__name__}.{f} %zu\\n", offsetof({t.__name__}, {f}));' for f, _ in t._fields_]
    src = tmp_path / "sizes.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "gemmtune_layers.h"\n'
                   'int main(void) {\n' + "\n".join(lines) + "\nreturn 0; }\n")
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-I", os.path.dirname(HEADER), str(src), "-o", str(exe)], check=True)
    want = dict(line.split() for line in
                subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines())
    for t in L.EXPORTS.values():
        assert ctypes.sizeof(t) == int(want[t.__name__])
        for f, _ in t._fields_:
            assert getattr(t, f).offset == int(want[f"{t.__name__}.{f}"])


# one valid argument structure of every entry point (gated layers of 5 rows, 16 → 24 columns)
M, K, N, E, TOP = 5, 16, 24, 4, 2
VALID = {
    "gt_linear": dict(M=M, N=N, K=K, dtype=1, act=19, out_dtype=1, X=AT, ldx=K, W=AT, ldw=2 * N, bias=AT,
                      R=AT, ldr=N, Y=AT, ldy=N, P=AT, ldp=2 * N),
    "gt_linear_backward": dict(M=M, N=N, K=K, dtype=1, act=19, dw_dtype=0, dY=AT, lddy=N, X=AT, ldx=K, W=AT,
                               ldw=2 * N, P=AT, ldp=2 * N, dX=AT, lddx=K, dW=AT, lddw=2 * N, db=AT),
    "gt_route": dict(T=M, E=E, k=TOP, groups=2, keep=1, dtype=1, score=1, renormalise=1, scale=1.0, logits=AT,
                     ldl=E, bias=AT, weights=AT, experts=AT, offsets=AT, order=AT, place=AT),
    "gt_route_backward": dict(T=M, E=E, k=TOP, dtype=1, score=0, renormalise=1, scale=1.0, logits=AT, ldl=E,
                              experts=AT, dweights=AT, dlogits=AT, lddl=E),
    "gt_experts": dict(T=M, D=K, H=N, E=E, k=TOP, dtype=1, act=18, X=AT, ldx=K, W1=AT, ldw1=2 * N,
                       sw1=2 * N * K, W2=AT, ldw2=K, sw2=N * K, b1=AT, b2=AT, R=AT, ldr=K, Y=AT, ldy=K, P=AT,
                       ldp=2 * N, weights=AT, offsets=AT, order=AT, place=AT),
    "gt_experts_backward": dict(T=M, D=K, H=N, E=E, k=TOP, dtype=1, act=18, dY=AT, lddy=K, X=AT, ldx=K, W1=AT,
                                ldw1=2 * N, sw1=2 * N * K, W2=AT, ldw2=K, sw2=N * K, b2=AT, P=AT, ldp=2 * N,
                                weights=AT, offsets=AT, order=AT, place=AT, dX=AT, lddx=K, dW1=AT, dW2=AT,
                                db1=AT, db2=AT, dweights=AT),
}
WRONG = {
    "gt_linear": [dict(M=-1), dict(N=0), dict(K=0), dict(M=1 << 31), dict(N=1 << 30), dict(dtype=2), dict(act=4),
                  dict(act=32), dict(out_dtype=-1), dict(X=None), dict(W=None), dict(Y=None), dict(ldx=K - 1),
                  dict(ldw=2 * N - 1), dict(ldr=N - 1), dict(ldy=N - 1), dict(ldp=2 * N - 1), dict(ldx=1 << 31),
                  dict(X=AT + 1), dict(W=AT + 1), dict(bias=AT + 1), dict(R=AT + 1), dict(Y=AT + 1),
                  dict(P=AT + 1), dict(out_dtype=0, Y=AT + 2), dict(out_dtype=0, R=AT, Y=AT),
                  dict(M=(1 << 31) - 1, ldx=1 << 20)],
    "gt_linear_backward": [dict(M=-1), dict(N=0), dict(K=0), dict(dtype=5), dict(act=20), dict(dw_dtype=2),
                           dict(dY=None), dict(P=None), dict(W=None), dict(X=None), dict(lddy=N - 1),
                           dict(ldx=K - 1), dict(ldw=N), dict(ldp=N), dict(lddx=K - 1), dict(lddw=N),
                           dict(dY=AT + 1), dict(dX=AT + 1), dict(dW=AT + 2), dict(db=AT + 2)],
    "gt_route": [dict(T=-1), dict(E=0), dict(E=1026), dict(k=0), dict(k=3), dict(k=65, E=1024, keep=2),
                 dict(groups=0), dict(groups=3), dict(keep=0), dict(keep=3), dict(dtype=2), dict(score=2),
                 dict(logits=None), dict(weights=None), dict(experts=None), dict(offsets=None), dict(order=None),
                 dict(place=None), dict(ldl=E - 1), dict(logits=AT + 1), dict(bias=AT + 2), dict(weights=AT + 2),
                 dict(T=1 << 30)],
    "gt_route_backward": [dict(T=-1), dict(E=0), dict(E=1025), dict(k=0), dict(k=5), dict(dtype=-1),
                          dict(score=-1), dict(logits=None), dict(experts=None), dict(dweights=None),
                          dict(dlogits=None), dict(ldl=E - 1), dict(lddl=E - 1), dict(dlogits=AT + 1),
                          dict(experts=AT + 2)],
    "gt_experts": [dict(T=-1), dict(D=0), dict(H=0), dict(E=0), dict(E=1025), dict(k=0), dict(k=65),
                   dict(T=1 << 30), dict(dtype=3), dict(act=64), dict(X=None), dict(W1=None), dict(W2=None),
                   dict(Y=None), dict(weights=None), dict(offsets=None), dict(order=None), dict(place=None),
                   dict(ldx=K - 1), dict(ldw1=N), dict(ldw2=K - 1), dict(ldr=1), dict(ldy=K - 1), dict(ldp=N),
                   dict(sw1=-1), dict(sw2=-8), dict(sw1=1 << 60), dict(X=AT + 1), dict(b1=AT + 1),
                   dict(order=AT + 2), dict(D=1 << 30, H=1 << 29, ldx=1 << 30, ldw1=1 << 30, ldw2=1 << 30,
                                            ldr=1 << 30, ldy=1 << 30, ldp=1 << 30)],
    "gt_experts_backward": [dict(T=-1), dict(D=0), dict(H=0), dict(E=1025), dict(k=65), dict(dtype=3),
                            dict(act=-1), dict(dY=None), dict(W2=None), dict(P=None), dict(weights=None),
                            dict(offsets=None), dict(order=None), dict(place=None), dict(W1=None), dict(X=None),
                            dict(lddy=K - 1), dict(ldx=K - 1), dict(ldw1=N), dict(ldw2=1), dict(ldp=N),
                            dict(lddx=K - 1), dict(sw2=-1), dict(dW1=AT + 1), dict(db1=AT + 2),
                            dict(dweights=AT + 1), dict(place=AT + 1)],
}


def args(L, name, **change):
    a = L.EXPORTS[name]()
    for f, v in {**VALID[name], **change}.items():
        setattr(a, f, v)
    return a


def call(L, name, a, ws=AT, ws_bytes=1 << 40):
    f = getattr(L.lib(), name)
    return f(ctypes.byref(a), None) if name in L.NO_SCRATCH else f(ctypes.byref(a), ws, ws_bytes, None)


def message(L):
    from paper_1909_10616_amd import gemmtune
    return gemmtune.lib().gt_last_error().decode()


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


@pytest.mark.parametrize("name,change", [("gt_linear", dict(X=AT + 2, act=3, K=4096, M=64, ldx=4096)),
                                         ("gt_linear_backward", {}), ("gt_route", dict(T=5000)),
                                         ("gt_experts", {}), ("gt_experts_backward", {})])
def test_scratch_too_small_or_misaligned(L, name, change):
    a = args(L, name, **change)
    need = L.workspace_bytes(name, a)
    assert need > 0
    assert call(L, name, a, AT, need - 1) == GT_ESMALL and str(need) in message(L)
    assert call(L, name, a, AT, 0) == GT_ESMALL
    assert call(L, name, a, None, need) == GT_EINVAL
    assert call(L, name, a, AT + 16, need) == GT_EINVAL


def test_no_rows_need_nothing(L):
    """Without rows the queries succeed, and a layer without gradients launches nothing."""
    for name in VALID:
        if name in L.NO_SCRATCH:
            continue
        a = args(L, name)
        setattr(a, "M" if hasattr(a, "M") else "T", 0)
        assert L.workspace_bytes(name, a) >= 0
    assert call(L, "gt_linear", args(L, "gt_linear", M=0, X=None, W=None, Y=None), None, 0) == 0


VALUES = [-(1 << 62), -7, -1, 0, 1, 2, 3, 5, 8, 16, 31, 64, 100, 256, 1000, 4096, 11008, 1 << 20, (1 << 31) - 1,
          1 << 31, 1 << 40, 1 << 62]


@pytest.mark.parametrize("name", [n for n in VALID if n != "gt_route_backward"])
def test_queries_survive_arbitrary_arguments(L, name):
    rng = random.Random(name)
    served = 0
    for i in range(4000):
        a = args(L, name)
        for f, t in a._fields_:
            wild = rng.random() < (0.15 if i % 2 else 0.5)
            if not wild:
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


def test_scratch_covers_large_serving_and_training_shapes(L):
    """The queries for shapes of every kind, from one row to the largest: a plan exists."""
    for m in (1, 2, 3, 4, 5, 16, 17, 64, 100, 999, 4096, 65536):
        for n in (1, 7, 64, 1021, 4096, 11008):
            for k in (1, 8, 777, 4096):
                for dtype in (0, 1):
                    for act in (0, 19):
                        w = 2 * n if act else n
                        a = args(L, "gt_linear", M=m, N=n, K=k, dtype=dtype, out_dtype=dtype, act=act, ldx=k,
                                 ldw=w, ldr=n, ldy=n, ldp=w)
                        assert 0 <= L.workspace_bytes("gt_linear", a) < 1 << 36


# ---------------------------------------------------------------------------
# the Python side
# ---------------------------------------------------------------------------

def test_cpu_tensors_are_refused(L):
    X, W = torch.zeros(4, 8), torch.zeros(8, 16)
    r = L.Route(torch.zeros(4, 2), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(5, dtype=torch.int32),
                torch.zeros(8, dtype=torch.int32), torch.zeros(4, 2, dtype=torch.int32))
    W1, W2 = torch.zeros(4, 8, 16), torch.zeros(4, 16, 8)
    for f in (lambda: L.gt_linear(X, W), lambda: L.gt_linear_backward(torch.zeros(4, 16), X, W),
              lambda: L.gt_route(X, 2), lambda: L.gt_route_backward(r.weights, X, r.experts),
              lambda: L.gt_experts(X, r, W1, W2),
              lambda: L.gt_experts_backward(X, X, r, W1, W2, torch.zeros(8, 16))):
        with pytest.raises(ValueError, match="GPU tensor"):
            f()
