"""The example of the layer operators: its gradients are autograd's, training lowers the
loss, and single tokens through a captured graph agree with the batch."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def X():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_1909_10616_amd import expert_layer
    return expert_layer


def test_gradients_are_autograds(X):
    """fp32 against autograd through a dense form of the same model, same choice of experts. Sums
    of at most 96 products and 40 tokens: 1e-5 of a gradient's largest value is ten times their
    rounding."""
    T, D, H, E, k, out = 40, 24, 32, 6, 2, 20
    m = X.ExpertLayer(D, H, E, k, out, torch.float32, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    m.low["b1"].copy_(torch.randn(E, 2 * H, generator=gen, device="cuda"))
    m.low["b2"].copy_(torch.randn(E, D, generator=gen, device="cuda"))
    x = torch.randn(T, D, generator=gen, device="cuda")
    dY = torch.randn(T, out, generator=gen, device="cuda")
    kept = {}
    Y = m.forward(x, keep=kept)
    got = m.backward(dY, kept)

    w = {n: t.detach().cpu().double().requires_grad_() for n, t in m.low.items()}
    xd, chosen = x.cpu().double(), kept["route"].experts.cpu().long()
    share = torch.softmax(xd @ w["router"], dim=1).gather(1, chosen)
    share = share / share.sum(1, keepdim=True)
    h = xd
    for s in range(k):
        e = chosen[:, s]
        p = (xd.unsqueeze(1) @ w["W1"][e]).squeeze(1) + w["b1"][e]
        a = torch.nn.functional.silu(p[:, :H]) * p[:, H:]
        h = h + share[:, s:s + 1] * ((a.unsqueeze(1) @ w["W2"][e]).squeeze(1) + w["b2"][e])
    want = h @ w["head"] + w["bias"]
    exact = want.detach()
    assert float((Y.cpu().double() - exact).abs().max()) <= 1e-5 * float(exact.abs().max())
    (want * dY.cpu().double()).sum().backward()
    for n, t in w.items():
        g = got[n].cpu().double()
        assert float((g - t.grad).abs().max()) <= 1e-5 * float(t.grad.abs().max()), n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_training_and_single_tokens(X, dtype):
    """The loss falls to less than a third; single tokens agree with the batch within the
    roundings between the layers (bf16: five of 2^-8 of values up to a few)."""
    losses, worst = X.main(["--tokens", "512", "--width", "64", "--hidden", "96", "--experts", "8", "--out", "40",
                            "--kinds", "4", "--steps", "150", "--serve", "16", "--dtype", dtype])
    assert losses[-1] < losses[0] / 3
    assert worst <= (0.1 if dtype == "bf16" else 1e-4)
