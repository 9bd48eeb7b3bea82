"""The RMS norm of rows whose length leaves fp32's range although their mean square root does not."""
import pytest
import torch

from paper_2609_13846_gb300 import dtp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROUND = 2.0 ** -24


def _rows(d, dtype):
    g = torch.Generator(device=DEV).manual_seed(d)
    x = torch.randn((7, d), generator=g, device=DEV)
    x[0] = 1e37
    x[1] *= 3e37
    x[2] = 0.0
    x[2, d // 2] = 3e38
    x[3] = -3.3e38
    x[4] = x[4].abs() * 1e19 + 1e19           # squares around fp32's largest
    x[5, : d // 2] = 2e38
    return x.to(dtype)


@pytest.mark.parametrize("d", [1, 24, 300, 1000, 1001, 2048, 4096, 8192, 8200, 1 << 20])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_beyond_the_range_of_their_squares(d, dtype):
    x = _rows(d, dtype)
    g = torch.Generator(device=DEV).manual_seed(1)
    gamma = 1.0 + 0.3 * torch.randn(d, generator=g, device=DEV)
    dy = (torch.randn(x.shape, generator=g, device=DEV) * 1e5).to(dtype)
    y, rms = dtp.rms_norm(x, gamma, eps=1e-6)
    dx, dgamma = dtp.rms_norm_backward(dy, x, gamma, rms)
    X, G, D = x.double(), gamma.double(), dy.double()
    R = (X.square().mean(-1) + 1e-6).sqrt()
    n = X / R[:, None]
    half, e = torch.finfo(dtype).eps / 2, (d / 32 + 24) * ROUND
    assert ((rms.double() - R).abs() <= e * R).all()
    assert ((y.double() - n * G).abs() <= (half + e) * 1.01 * (n * G).abs() + 1e-38).all()
    dn = D * G
    want = (dn - n * (dn * n).mean(-1, keepdim=True)) / R[:, None]
    size = (dn.abs() + n.abs() * (dn * n).abs().mean(-1, keepdim=True)) / R[:, None]
    # 1 / rms may be a subnormal number: off by 2^-150 of at least 2^-128.1, in three places
    assert ((dx.double() - want).abs() <= half * want.abs() + (4 * e + 3 * 2.0 ** -21) * size + 1e-38).all()
    assert ((dgamma.double() - (D * n).sum(0)).abs() <= (23 + d / 32) * ROUND * (D * n).abs().sum(0) + 2.0 ** -21 * (D * n).abs().sum(0)).all()


@pytest.mark.parametrize("d", [24, 1001, 4096, 8200])
@pytest.mark.parametrize("eps", [1e30, 2e38, 3.4e38])
def test_an_eps_of_any_size_counts(d, eps):
    """Mean squares, eps and their sums on both sides of fp32's largest number."""
    g = torch.Generator(device=DEV).manual_seed(d)
    x = torch.rand((9, d), generator=g, device=DEV) + 0.5
    x *= torch.tensor([0.0, 1e10, 1e15, 0.9e19, 1.2e19, 1.7e19, 1e20, 1e30, 1e37], device=DEV)[:, None]
    gamma = torch.ones(d, device=DEV)
    y, rms = dtp.rms_norm(x, gamma, eps=eps)
    eps = float(torch.tensor(eps))
    R = (x.double().square().mean(-1) + eps).sqrt()
    n = x.double() / R[:, None]
    e = (d / 32 + 24) * ROUND
    assert ((rms.double() - R).abs() <= e * R).all()
    assert ((y.double() - n).abs() <= (ROUND + e) * 1.01 * n.abs() + 1e-38).all()
