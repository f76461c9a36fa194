"""Where the layer operators' sizes end, on the CPU: the last that is served and the first that is
refused."""
import ctypes

import pytest

from test_layers_host import GT_EINVAL, L, args  # noqa: F401


@pytest.mark.parametrize("name,most", [("gt_experts", 1 << 29), ("gt_experts_backward", 1 << 29),
                                       ("gt_route", 1 << 31)])
def test_entries(L, name, most):  # noqa: F811
    n = ctypes.c_int64()
    query = getattr(L.lib(), name + "_workspace")
    for T, k in ((most // 2, 2), (most // 2 - 1, 2), (most - 1, 1)):
        a = args(L, name, T=T, k=k)
        served = T * k < most
        assert query(ctypes.byref(a), ctypes.byref(n)) == (0 if served else GT_EINVAL), (T, k)
        if served:
            assert n.value >= 0


@pytest.mark.parametrize("name", ["gt_linear", "gt_linear_backward"])
def test_extents(L, name):  # noqa: F811
    n = ctypes.c_int64()
    query = getattr(L.lib(), name + "_workspace")
    last = (1 << 31) - 1
    for field, lds in (("M", ()), ("K", ("ldx", "lddx"))):
        for value, served in ((last, True), (last + 1, False)):
            have = {f for f, _ in L.EXPORTS[name]._fields_}
            a = args(L, name, **{field: value}, **{ld: min(value, last) for ld in lds if ld in have})
            assert query(ctypes.byref(a), ctypes.byref(n)) == (0 if served else GT_EINVAL), (field, value)
