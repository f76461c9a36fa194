"""Which gradients of the norm are asked for, without a GPU: names that are none are refused before anything
else is looked at."""
import pytest
import torch


@pytest.fixture(scope="module")
def L():
    from paper_1909_10616_amd import layers
    layers.lib()
    return layers


@pytest.mark.parametrize("need", [("dx",), ("dweights",), ("dX", "dW"), "dX, dweight", "dXdweight", ("",), "", [None],
                                  ("dX", "residual")], ids=str)
def test_unknown_names_are_refused(L, need):
    X, v = torch.zeros(4, 128), torch.zeros(4)
    with pytest.raises(ValueError, match="need"):
        L.gt_norm_backward(X, X, v, v, need=need)


@pytest.mark.parametrize("need", [(), [], "dX", "dweight", ("dX",), ["dweight", "dX"], {"dX"}, ("dX", "dweight", "dbias"),
                                  "dbias"], ids=str)
def test_names_that_are_gradients_pass(L, need):
    X, v = torch.zeros(4, 128), torch.zeros(4)
    with pytest.raises(ValueError, match="GPU tensor"):   # (the next check)
        L.gt_norm_backward(X, X, v, v, need=need)
