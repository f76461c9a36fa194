"""What the layer operators' Python functions refuse: wrong types, shapes,
strides and devices, by name, before anything runs."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_1909_10616_amd import layers
    layers.lib()
    return layers


def z(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype, device="cuda")


def test_linear(L):
    X, W = z(4, 8), z(8, 16)
    wrong = [
        (dict(W=z(9, 16)), "W has shape"), (dict(W=z(8, 16, dtype=BF16)), "W must be"),
        (dict(X=z(4, 8, dtype=torch.float16)), "float32 or bfloat16"), (dict(X=z(4, 4, 8)), "2 dimensions"),
        (dict(W=z(16, 8).t()), "rows of W"), (dict(bias=z(15)), "bias has shape"),
        (dict(bias=z(32)[::2]), "rows of bias"), (dict(bias=z(16).cpu()), "bias must be a GPU tensor"),
        (dict(residual=z(4, 15)), "residual has shape"), (dict(Y=z(4, 17)), "Y has shape"),
        (dict(P=z(4, 15)), "P has shape"), (dict(act="tanh"), "unknown activation"),
        (dict(W=z(8, 15), gated=True), "even number"), (dict(X=z(1, 8).expand(4, 8)), "overlap"),
        (dict(workspace=torch.zeros(8, dtype=torch.uint8)), None),
    ]
    for change, match in wrong:
        a = {"X": X, "W": W, **change}
        if match is None:     # (no scratch is needed here, so none is looked at)
            L.gt_linear(**a)
            continue
        with pytest.raises(ValueError, match=match):
            L.gt_linear(**a)


def test_linear_backward(L):
    a = dict(dY=z(4, 16), X=z(4, 8), W=z(8, 16), P=z(4, 16), act="silu")
    L.gt_linear_backward(**a)
    for change, match in [(dict(P=None), "needs P"), (dict(dY=z(4, 15)), "dY has shape"),
                          (dict(P=z(4, 15)), "P has shape"), (dict(dX=z(4, 9)), "dX has shape"),
                          (dict(dX=z(4, 8, dtype=BF16)), "dX must be"), (dict(db=z(15)), "db has shape"),
                          (dict(db=z(16, dtype=BF16)), "db must be"), (dict(gated=True, W=z(8, 17)), "even number")]:
        with pytest.raises(ValueError, match=match):
            L.gt_linear_backward(**{**a, **change})


def test_route(L):
    x = z(5, 8)
    r = L.gt_route(x, 2)
    for kw, match in [(dict(k=0), "k is 0"), (dict(k=9), "k is 9"), (dict(score="max"), "unknown score"),
                      (dict(bias=z(7)), "bias has shape"), (dict(bias=z(8, dtype=BF16)), "bias must be")]:
        with pytest.raises(ValueError, match=match):
            L.gt_route(x, **{"k": 2, **kw})
    for kw in (dict(groups=3), dict(groups=4, keep=5), dict(groups=4, keep=1, k=3)):
        with pytest.raises(L.gt.GemmTuneError, match="gt_route"):
            L.gt_route(x, **{"k": 2, **kw})
    with pytest.raises(ValueError, match="dweights has shape"):
        L.gt_route_backward(z(5, 3), x, r.experts)
    with pytest.raises(ValueError, match="experts must be"):
        L.gt_route_backward(r.weights, x, r.experts.float())


def test_experts(L):
    r = L.gt_route(z(5, 4), 2)
    a = dict(X=z(5, 8), route=r, W1=z(4, 8, 16), W2=z(4, 16, 8))
    L.gt_experts(**a)
    for change, match in [(dict(W1=z(3, 8, 16)), "W1 has shape"), (dict(W2=z(4, 15, 8)), "W2 has shape"),
                          (dict(W1=z(4, 16, 8).transpose(1, 2)), "rows of W1"), (dict(b1=z(4, 15)), "b1 has shape"),
                          (dict(b2=z(4, 9)), "b2 has shape"), (dict(X=z(6, 8)), "weights has shape"),
                          (dict(P=z(9, 16)), "P has shape"), (dict(gated=True, W1=z(4, 8, 15)), "even number"),
                          (dict(route=r._replace(order=r.order[1:])), "order has shape"),
                          (dict(route=r._replace(place=r.place.long())), "place must be"),
                          (dict(W1=z(4, 8, 16, dtype=BF16)), "W1 must be")]:
        with pytest.raises(ValueError, match=match):
            L.gt_experts(**{**a, **change})
    b = dict(dY=z(5, 8), P=z(10, 16), **a)
    L.gt_experts_backward(**b)
    for change, match in [(dict(dY=z(5, 9)), "dY has shape"), (dict(P=z(10, 15)), "P has shape"),
                          (dict(b2=z(4, 9)), "b2 has shape")]:
        with pytest.raises(ValueError, match=match):
            L.gt_experts_backward(**{**b, **change})


def test_misaligned_to_its_elements(L):
    raw = torch.zeros(4 * 8 * 4 + 2, dtype=torch.uint8, device="cuda")
    a = L.gt_linear_args(4, 8, 8, 0, 0, 0, 0, raw.data_ptr() + 2, 8, z(8, 8).data_ptr(), 8, None, None, 8,
                         z(4, 8).data_ptr(), 8, None, 8)
    with pytest.raises(L.gt.GemmTuneError, match="aligned"):
        L.workspace_bytes("gt_linear", a)
