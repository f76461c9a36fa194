"""More sizes for the layer operators' kernels of a few rows and of many tokens: the
definitions, bounds and frames of test_gpu_layers at extents that end inside a
lane's share of experts, a quad of columns or a step of k."""
import pytest

import test_gpu_layers as base
from test_gpu_layers import BF16, F32, IDS, L  # noqa: F401

pytestmark = pytest.mark.gpu

ROUTES = [
    # T, E, k, score, groups, keep, bias, renormalise
    (200, 30, 12, "softmax", 1, 1, True, True), (150, 100, 9, "sigmoid", 1, 1, False, False),
    (90, 255, 16, "softmax", 1, 1, True, False), (101, 192, 6, "sigmoid", 3, 2, True, True),
    (99, 96, 8, "softmax", 3, 2, False, False), (67, 256, 16, "softmax", 2, 1, True, True),
    (130, 64, 5, "sigmoid", 16, 4, True, False), (515, 5, 5, "softmax", 1, 1, False, True),
    (2050, 128, 1, "softmax", 16, 16, False, False), (70, 256, 17, "sigmoid", 1, 1, False, True),
    (80, 240, 8, "sigmoid", 5, 3, True, True),
]


@pytest.mark.parametrize("kind", ["plain", "ties", "holes", "far"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS.get)
@pytest.mark.parametrize("case", ROUTES, ids=str)
def test_route(L, case, dtype, kind):  # noqa: F811
    base.test_route(L, case, dtype, kind)


@pytest.mark.parametrize("pad", [0, 8, 5])
@pytest.mark.parametrize("shape", [(5, 1, 1), (7, 65, 33), (16, 64, 16), (17, 100, 300), (40, 33, 1000),
                                   (64, 200, 77), (6, 12, 2100), (31, 129, 512), (1, 200, 4100), (3, 70, 5000), (2, 129, 3001),
                                   (4, 64, 2056)], ids=str)
@pytest.mark.parametrize("dtype", [BF16, F32], ids=IDS.get)
def test_linear(L, dtype, shape, pad):  # noqa: F811
    base.test_linear(L, dtype, shape, pad)


@pytest.mark.parametrize("case", [(BF16, 9, 264, 4096), (F32, 9, 260, 2048), (F32, 33, 70, 4100), (BF16, 48, 130, 2056)],
                         ids=lambda c: f"{IDS[c[0]]}-{c[1]}x{c[2]}x{c[3]}")
def test_linear_whole_numbers(L, case):  # noqa: F811
    base.test_linear_whole_numbers(L, case)


@pytest.mark.parametrize("holes", [False, True])
@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("case", [(48, 6, 2, 72, 40), (100, 8, 1, 130, 66), (37, 3, 2, 33, 129), (2, 3, 2, 4100, 40), (1, 4, 2, 520, 2056)], ids=str)
@pytest.mark.parametrize("dtype", [BF16, F32], ids=IDS.get)
def test_experts_and_their_gradients(L, dtype, case, pad, holes):  # noqa: F811
    base.test_experts_and_their_gradients(L, dtype, case, pad, holes)


@pytest.mark.parametrize("case", [(40, 200, 3, 64, 48), (120, 300, 4, 72, 40), (300, 130, 3, 40, 24)], ids=str)
@pytest.mark.parametrize("dtype", [BF16, F32], ids=IDS.get)
def test_many_experts(L, dtype, case):  # noqa: F811
    base.test_experts_and_their_gradients(L, dtype, case, 3, True)
