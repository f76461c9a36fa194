"""Results in another type than the operands': fp32 for bf16 operands, and nothing else. The library
refuses a bf16 result of fp32 operands before any launch, and so does the binding, by name."""
import ctypes

import pytest
import torch

from test_layers_host import GT_EINVAL, L, args, call, message  # noqa: F401

F32, BF16 = 0, 1


@pytest.mark.parametrize("name,field,change", [("gt_linear", "out_dtype", dict(R=None)),
                                               ("gt_linear_backward", "dw_dtype", {})])
def test_library(L, name, field, change):  # noqa: F811
    n = ctypes.c_int64()
    query = getattr(L.lib(), name + "_workspace")
    for dtype, out, served in ((F32, F32, True), (BF16, BF16, True), (BF16, F32, True), (F32, BF16, False)):
        a = args(L, name, dtype=dtype, **{field: out}, **change)
        assert query(ctypes.byref(a), ctypes.byref(n)) == (0 if served else GT_EINVAL)
        if not served:
            assert "fp32" in message(L)
            assert call(L, name, a) == GT_EINVAL


@pytest.mark.gpu
def test_binding(L):  # noqa: F811
    def z(*shape, dtype=torch.float32):
        return torch.zeros(*shape, dtype=dtype, device="cuda")

    X, W, bf16 = z(40, 72), z(72, 96), torch.bfloat16
    with pytest.raises(ValueError, match="Y must be torch.float32"):
        L.gt_linear(X, W, Y=z(40, 96, dtype=bf16))
    with pytest.raises(ValueError, match="dW must be torch.float32"):
        L.gt_linear_backward(z(40, 96), X, W, dW=z(72, 96, dtype=bf16))
    Y = z(40, 96)
    assert L.gt_linear(X.to(bf16), W.to(bf16), Y=Y) is Y
    dW = z(72, 96)
    assert L.gt_linear_backward(z(40, 96, dtype=bf16), X.to(bf16), W.to(bf16), dW=dW)[1] is dW
