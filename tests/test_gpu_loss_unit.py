"""dZ in units of the largest dloss, over more tokens than a weight gradient's run."""
import pytest
import torch

from paper_2609_13846_gb300 import dtp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("T", [20_000, (1 << 18) + 4097])
@pytest.mark.parametrize("padding", [0.0, 0.5])
def test_a_means_gradient_is_not_rounded_the_same_way_in_every_row(T, padding):
    """dloss is the same in all rows and lies half a bf16 step from its neighbours: rounded to bf16 it is off by 0.37%, and so would
    both gradients be along themselves.  In units of itself it is 1: what is left is the target's p - 1, whose p of about 1/4096
    is lost against 1 (2.4e-4, 3e-4 with the probabilities' spread), and roundings of random sign; 1e-3 holds them."""
    d, V = 64, 4096
    g = torch.Generator(device=DEV).manual_seed(5)
    x = torch.randn((T, d), generator=g, device=DEV).to(torch.bfloat16)
    w = (torch.randn((V, d), generator=g, device=DEV) * 0.05).to(torch.bfloat16)
    y = torch.randint(0, V, (T,), generator=g, device=DEV)
    y[torch.rand(T, generator=g, device=DEV) < padding] = -100
    size = 2.0 ** -18 * (1.0 + 2.0 ** -8 * 0.96)
    dloss = torch.full((T,), size, device=DEV)
    assert abs(float(dloss[0].to(torch.bfloat16)) / size - 1.0) > 3.5e-3
    _, lse = dtp.linear_cross_entropy(x, w, y)
    dx, dw = dtp.linear_cross_entropy_backward(dloss, x, w, y, lse, check=True)
    W = w.double()
    want, top, bottom = torch.zeros_like(W), 0.0, 0.0
    for t in range(0, T, 1 << 15):
        X, at = x[t:t + (1 << 15)].double(), y[t:t + (1 << 15)]
        live = (at != -100).double()[:, None]
        dz = torch.softmax(X @ W.t(), 1)
        dz.scatter_add_(1, torch.where(at == -100, 0, at)[:, None], -torch.ones_like(live))
        dz *= size * live
        want += dz.t() @ X
        ref = dz @ W
        top += float((ref * dx[t:t + (1 << 15)].double()).sum())
        bottom += float(ref.square().sum())
    assert abs(top / bottom - 1.0) <= 1e-3
    assert abs(float((want * dw.double()).sum() / want.square().sum()) - 1.0) <= 1e-3
