"""Which form the 8-bit products of the tests take, without a GPU: every form there is, among them."""
import ctypes

import pytest

from layers8_forms import FORMS, form
from test_layers8_host import L, args  # noqa: F401


def arguments(L, M, N, K, gated, out, **change):  # noqa: F811
    ld, kb, t = (K + 15) // 16 * 16, -(-K // 128), int(out == "bf16")
    return args(L, "gt_linear_fp8", **{**dict(M=M, N=N, K=K, act=L.GATED if gated else 0, dtype=t, out_dtype=t, ldx=ld,
                                              ldw=ld, ldsx=kb, ldsw=kb, bias=None, R=None, ldy=N), **change})


@pytest.mark.parametrize("case", FORMS, ids=str)
@pytest.mark.parametrize("wblock", [1, 128])
def test_a_sizes_form(L, case, wblock):  # noqa: F811
    took, fp32 = form(L, arguments(L, *case, wblock=wblock))
    assert took == FORMS[case]
    assert fp32 == (took[0] > 0 or case[4] == "f32")


def test_every_form_is_among_them():
    have = {(rows, tile, slices > 1, gated, out) for (_, _, _, gated, out), (rows, tile, slices) in FORMS.items()}
    for gated in (False, True):
        for rows in (16, 32) if gated else (16, 32, 64):
            assert (rows, -1, False, gated, "bf16") in have
        for tile in (0, 1, 2):
            for sliced in (False, True):
                assert (0, tile, sliced, gated, "bf16") in have
    # (a result in fp32 has no 256×256 tile)
    assert {(t, s) for _, t, s, _, out in have if out == "f32"} == {(-1, False), (1, False), (1, True), (2, False), (2, True)}


def test_a_query_of_wrong_arguments_is_refused(L):  # noqa: F811
    f = L.lib().gt_linear_fp8_form
    out = (ctypes.c_int32 * 4)(*[7] * 4)
    assert f(None, out) == -1 and f(ctypes.byref(args(L, "gt_linear_fp8", K=0)), out) == -1
    assert f(ctypes.byref(args(L, "gt_linear_fp8")), None) == -1 and list(out) == [7] * 4
