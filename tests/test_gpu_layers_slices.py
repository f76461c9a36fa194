"""Experts of few rows whose up product is cut into K slices while its rows are padded to whole
16-byte chunks: small whole numbers, exact in any order, with scratch of exactly the
size asked for and a frame behind it."""
import pytest
import torch

from test_gpu_layers import BF16, F32, IDS, L  # noqa: F401

pytestmark = pytest.mark.gpu


def scratch(L, X, r, W1, W2, Y, P, act, gated):  # noqa: F811
    """The bytes gt_experts asks for."""
    (T, D), (E, H, _), k = X.shape, W2.shape, r.weights.shape[1]
    wide = W1.shape[2]
    ptr = [t.data_ptr() for t in (X, W1, W2, Y, P, *r)]
    a = L.gt_experts_args(T, D, H, E, k, L._type(X, "X"), L._act(act, gated), ptr[0], D, ptr[1], wide, D * wide,
                          ptr[2], D, H * D, None, None, None, D, ptr[3], D, ptr[4], wide, ptr[5], ptr[7],
                          ptr[8], ptr[9])
    return L.workspace_bytes("gt_experts", a)


def up(v, m):
    return (v + m - 1) // m * m


# T, E, k, D, then H of every remainder by 8 that leaves an empty quad, and the others
FEW = [(1, 8, 2, 1814), (2, 4, 1, 2048), (3, 6, 2, 2048), (4, 36, 1, 4100)]
SLIM = [(16, 4, 1, 4100), (24, 4, 2, 1814), (48, 8, 2, 2048)]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("H", [129, 130, 131, 132, 133, 136, 516, 1001, 1004])
@pytest.mark.parametrize("case", FEW + SLIM, ids=str)
@pytest.mark.parametrize("dtype", [BF16, F32], ids=IDS.get)
def test_experts_whole_numbers(L, dtype, case, H, gated):  # noqa: F811
    T, E, k, D = case
    print(f"experts in slices {dtype} {case} H {H} gated {gated}", flush=True)
    gen = torch.Generator().manual_seed(T * H + gated)
    r = L.gt_route(torch.randn(T, E, generator=gen).cuda(), k)
    r = r._replace(weights=torch.full_like(r.weights, 0.5))
    wide = H * (2 if gated else 1)
    # eight ones a token, spread over D: |P| ≤ 8 and |act(gate)·up| ≤ 64, whole in bf16
    X = torch.zeros(T, D)
    X.scatter_(1, torch.rand(T, D, generator=gen).topk(8, dim=1).indices, 1.0)
    X = X.to(dtype).cuda()
    gen = torch.Generator(device="cuda").manual_seed(T * H + gated)
    W1 = torch.randint(-1, 2, (E, D, wide), generator=gen, device="cuda").to(dtype)
    W2 = torch.randint(-1, 2, (E, H, D), generator=gen, device="cuda").to(dtype)
    Y = torch.empty(T, D, dtype=dtype, device="cuda")
    P = torch.empty(T * k, wide, dtype=dtype, device="cuda")
    need = scratch(L, X, r, W1, W2, Y, P, "relu", gated)
    if case in FEW:   # the slices of the up product are there
        vec, part = 16 // X.element_size(), T * k * up(H, 4) * (2 if gated else 1) * 4
        rows = up(T * k * up(H, vec) * X.element_size(), 256) + up(T * k * up(D, 4) * 4, 256)
        assert need - rows >= 2 * part
    ws = torch.full((need + 512,), 0x5a, dtype=torch.uint8, device="cuda")
    L.gt_experts(X, r, W1, W2, act="relu", gated=gated, Y=Y, P=P, workspace=ws[:need])
    assert bool((ws[need:] == 0x5a).all())

    chosen, place = r.experts.long(), r.place.long()
    want = torch.zeros(T, D, device="cuda")
    for s in range(k):
        p = torch.bmm(X.float().unsqueeze(1), W1[chosen[:, s]].float()).squeeze(1)
        assert torch.equal(P[place[:, s]].float(), p)
        h = p[:, :H].relu() * p[:, H:] if gated else p.relu()
        want += 0.5 * torch.bmm(h.unsqueeze(1), W2[chosen[:, s]].float()).squeeze(1)
    assert torch.equal(Y, want.to(dtype))
    again = L.gt_experts(X, r, W1, W2, act="relu", gated=gated)
    assert torch.equal(again, Y)
