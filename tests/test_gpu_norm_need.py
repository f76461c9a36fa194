"""Which gradients of the norm a call gives."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_1909_10616_amd import layers
    layers.lib()
    return layers


@pytest.mark.parametrize("need,bias,given", [("dX", False, "dX"), ("dX", True, "dX dbias"), ("dbias", False, "dbias"),
                                             (["dweight"], False, "dweight"), ((), True, "dbias"), ((), False, ""),
                                             ({"dX", "dbias"}, False, "dX dbias"),
                                             (("dX", "dweight", "dbias"), False, "dX dweight dbias")], ids=str)
@pytest.mark.parametrize("M", [9, 1100])
def test_what_is_given(L, M, need, bias, given):
    gen = torch.Generator().manual_seed(M)
    X, dY = (torch.randn(M, 200, generator=gen).cuda() for _ in range(2))
    mean, rstd = torch.empty(2, M, device="cuda")
    L.gt_norm(X, mean=mean, rstd=rstd)
    want = L.gt_norm_backward(dY, X, mean, rstd)
    got = L.gt_norm_backward(dY, X, mean, rstd, need=need, bias=bias)
    torch.cuda.synchronize()
    for name, a, b in zip(got._fields, got, want):
        assert (a is not None) == (name in given.split())
        assert a is None or torch.equal(a, b)
