"""Sizes that reach every form of the 8-bit products: tiles of 256×256 (0), 128×128 (1) and 64×64 (2),
in one piece and in K slices, and the kernels of 16, 32 and 64 rows, with a bf16 result and
with one in fp32, gated and not."""
import ctypes

import torch

# M, N, K, gated, type of Y: (rows a workgroup or 0, tile or −1, K slices)
FORMS = {
    (4100, 2100, 77, False, "bf16"): (0, 0, 1), (2100, 4100, 520, False, "bf16"): (0, 0, 1),
    (2500, 5000, 130, False, "bf16"): (0, 0, 1), (4096, 4096, 1000, False, "bf16"): (0, 0, 1),
    (2050, 2056, 333, True, "bf16"): (0, 0, 1), (2000, 2300, 4000, True, "bf16"): (0, 0, 1),
    (2304, 2048, 1021, True, "bf16"): (0, 0, 1),
    (2853, 130, 63071, False, "bf16"): (0, 0, 16), (2805, 65, 62757, True, "bf16"): (0, 0, 16),
    (2050, 2056, 136, False, "bf16"): (0, 1, 1), (1999, 2623, 3457, False, "bf16"): (0, 1, 1),
    (900, 3100, 900, True, "bf16"): (0, 1, 1), (1000, 2304, 707, True, "bf16"): (0, 1, 1),
    (4690, 197, 3849, False, "bf16"): (0, 1, 4), (79, 4635, 4346, True, "bf16"): (0, 1, 4),
    (515, 1021, 333, False, "bf16"): (0, 2, 1), (515, 1021, 333, True, "bf16"): (0, 2, 1),
    (600, 640, 391, True, "bf16"): (0, 2, 1),
    (300, 2050, 4000, False, "bf16"): (0, 2, 4), (300, 2050, 4000, True, "bf16"): (0, 2, 2),
    (1, 4096, 1021, False, "bf16"): (16, -1, 1), (17, 16, 139, False, "bf16"): (16, -1, 1),
    (64, 700, 4096, False, "bf16"): (16, -1, 1), (1, 1003, 777, True, "bf16"): (16, -1, 1),
    (17, 16, 260, True, "bf16"): (16, -1, 1), (3033, 18, 141, False, "bf16"): (32, -1, 1),
    (17, 2980, 258, True, "bf16"): (32, -1, 1), (35, 3081, 294, False, "bf16"): (64, -1, 1),
    (2050, 2056, 333, False, "f32"): (0, 1, 1), (2050, 2056, 333, True, "f32"): (0, 1, 1),
    (600, 2050, 5003, False, "f32"): (0, 1, 4), (1000, 1300, 777, True, "f32"): (0, 2, 1),
    (300, 300, 20001, False, "f32"): (0, 2, 16), (300, 2050, 4000, True, "f32"): (0, 2, 2),
    (35, 3081, 294, False, "f32"): (64, -1, 1), (17, 2980, 258, True, "f32"): (32, -1, 1),
}
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def form(L, a):
    """What a call with these arguments takes: (rows, tile, K slices), and whether its sums are fp32's."""
    out = (ctypes.c_int32 * 4)()
    assert L.lib().gt_linear_fp8_form(ctypes.byref(a), out) == 0
    return tuple(out[:3]), bool(out[3])


def form_of(L, X, W, Y, gated, **more):
    """The same of a call of the binding."""
    (M, K), wide = X.values.shape, W.values.shape[0]
    out = 1 if Y.dtype is torch.bfloat16 else 0
    a = L.gt_linear_fp8_args(M, wide // 2 if gated else wide, K, out, L.GATED if gated else 0, out, 0, 0, 1, 128, 0,
                             X.values.data_ptr(), X.values.stride(0), X.scales.data_ptr(), X.scales.stride(0),
                             W.values.data_ptr(), W.values.stride(0), W.scales.data_ptr(), W.scales.stride(0),
                             None, None, 0, Y.data_ptr(), Y.stride(0))
    if W.scales.shape[0] == wide:
        a.wblock = 1
    for name, v in more.items():
        setattr(a, name, v)
    return form(L, a)
