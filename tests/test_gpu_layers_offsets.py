"""Offsets that leave the rows or do not ascend: experts that overlap or have no rows. Which rows
such lists name is the caller's affair; every access stays inside the operands and the scratch."""
import pytest
import torch

from test_gpu_layers import BF16, F32, IDS, Frame, L, routed  # noqa: F401

pytestmark = pytest.mark.gpu

CHANGES = {"far": {2: 1 << 30}, "negative": {3: -(1 << 30)}, "descending": {1: 9, 2: 7, 3: 5, 4: 3, 5: 1},
           "to and fro": {1: 1 << 30, 2: 0, 3: 1 << 30, 4: 0, 5: 1 << 30}}


@pytest.mark.parametrize("change", CHANGES)
@pytest.mark.parametrize("T,D,H", [(40, 72, 64), (3, 2048, 40), (900, 136, 260)])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=IDS.get)
def test_experts_and_their_gradients(L, dtype, T, D, H, change):  # noqa: F811
    E, k = 6, 2
    print(f"offsets {change} {dtype} {T} {D} {H}", flush=True)
    f = Frame(T, 8)
    r = routed(L, f, T, E, k, False)
    for at, value in CHANGES[change].items():
        r.offsets[at] = value
    X, dY = f.normal(dtype, T, D), f.normal(dtype, T, D)
    W1, W2 = f.normal(dtype, E, D, H), f.normal(dtype, E, H, D)
    b1, b2 = f.normal(dtype, E, H).contiguous(), f.normal(dtype, E, D).contiguous()
    Y, P = f.output(dtype, T, D), f.output(dtype, T * k, H)
    ws = torch.full((64 << 20,), 0, dtype=torch.uint8, device="cuda")
    L.gt_experts(X, r, W1, W2, b1=b1, b2=b2, act="silu", Y=Y, P=P, workspace=ws)
    g = L.gt_experts_backward(dY, X, r, W1, W2, P, b2=b2, act="silu", workspace=ws)
    torch.cuda.synchronize()
    f.untouched()
    # an expert whose offsets leave it no rows has no gradient
    lo = r.offsets.clamp(0, T * k).cpu()
    for e in range(E):
        if lo[e + 1] <= lo[e]:
            assert not g.dW1[e].any() and not g.dW2[e].any()
            assert not g.db1[e].any() and not g.db2[e].any()
