"""The norm and its gradients of more rows than workgroups, so that each takes several, in every width's
kernel."""
import pytest
import torch

import layers8_plain as ref8
import layers_plain as ref
from test_gpu_layers8 import BF16, F32, IDS, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_1909_10616_amd import layers
    layers.lib()
    return layers


# widths of each kernel, and more rows than its workgroups take at once
MANY = [(8300, 100, 8192), (8300, 1000, 8192), (2100, 1500, 2048), (1400, 4001, 1280), (600, 6000, 512), (300, 12000, 256),
        (4100, 16400, 4096)]


@pytest.mark.parametrize("case", MANY, ids=str)
@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS.get)
def test_rows_after_a_workgroups_first(L, dtype, case):
    """Rows that repeat the first ones, one workgroup's turn later, have their bits; those have their values."""
    M, N, turn = case
    some = 4
    x = rows(torch.Generator().manual_seed(N), some, N, dtype)
    X = torch.zeros(M, N, dtype=dtype, device="cuda")
    X[:some] = x.cuda()
    X[turn:turn + some] = x.cuda()
    X[M - some:] = x.cuda()
    w, b = (torch.randn(N, generator=torch.Generator().manual_seed(i)).cuda() for i in (1, 2))
    mean, rstd = torch.empty(2, M, device="cuda")
    Y = L.gt_norm(X, w, b, mean=mean, rstd=rstd)
    q = L.gt_norm_fp8(X, w, b, code="e5m2")
    torch.cuda.synchronize()
    want, wmean, wrstd = ref8.norm(X[:some], w, b, 1e-5, dtype)
    ref.check(Y[:some], want, "Y")
    ref.check(mean[:some], wmean, "mean")
    ref.check(rstd[:some], wrstd, "rstd")
    for at in (slice(turn, turn + some), slice(M - some, M)):
        for t in (Y, mean, rstd, q.values.view(torch.uint8), q.scales):
            assert torch.equal(t[at], t[:some])
    zero = torch.ones(M, dtype=torch.bool, device="cuda")
    zero[:some] = zero[turn:turn + some] = zero[M - some:] = False
    assert bool((Y[zero] == b.to(dtype)).all()) and not bool(mean[zero].any())


@pytest.mark.parametrize("shape", [(1100, 1500), (1300, 2041), (1100, 2048), (2200, 300)], ids=str)
@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS.get)
def test_gradients_of_many_rows(L, dtype, shape):
    """Their sums in the rows' launch, a workgroup with several rows: with R, of statistics that are checked."""
    M, N = shape
    gen = torch.Generator().manual_seed(M + N)
    X, dY, R = (rows(gen, M, N, dtype).cuda() for _ in range(3))
    w = torch.randn(N, generator=gen).cuda()
    mean, rstd = torch.empty(2, M, device="cuda")
    L.gt_norm(X, w, mean=mean, rstd=rstd)
    g = L.gt_norm_backward(dY, X, mean, rstd, weight=w, residual=R)
    torch.cuda.synchronize()
    _, wmean, wrstd = ref8.norm(X, w, None, 1e-5, dtype)
    ref.check(mean, wmean, "mean")
    ref.check(rstd, wrstd, "rstd")
    for have, want, name in zip(g, ref8.norm_backward(dY, X, mean, rstd, w, R, dtype), ("dX", "dw", "db")):
        ref.check(have, want, name)
