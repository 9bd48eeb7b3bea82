"""A vocabulary of which all but a few tokens are masked by weights of -inf: what does not count stays out of the gradients."""
import pytest
import torch

from paper_2609_13846_gb300 import dtp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
IGNORE = -100
BF16, F32 = torch.bfloat16, torch.float32
D, V, KEPT = 64, 500, (7, 130, 499)


def _inputs(T, dtype, padding):
    """(x, w, y, dloss): x[:, 0] = 1 and w[:, 0] = -inf but for KEPT; tokens of padding hold NaNs."""
    g = torch.Generator(device=DEV).manual_seed(T)
    x = torch.randn((T, D), generator=g, device=DEV).to(dtype)
    w = (torch.randn((V, D), generator=g, device=DEV) * 0.2).to(dtype)
    x[:, 0] = 1.0
    kept = torch.tensor(KEPT, device=DEV)
    w[:, 0] = float("-inf")
    w[kept, 0] = 0.0
    y = kept[torch.randint(0, len(KEPT), (T,), generator=g, device=DEV)]
    off = torch.rand(T, generator=g, device=DEV) < padding
    y[off] = IGNORE
    x[off] = float("nan")
    return x, w, y, torch.rand(T, generator=g, device=DEV) / T


def _reference(x, w, y, dloss):
    """(dZ, X, W) in 64 bits, X's padding and W's masked column taken out."""
    live = y != IGNORE
    X = torch.where(live[:, None], x.double(), 0.0)
    W = w.double()
    mask = torch.isinf(W[:, 0])
    W[:, 0] = 0.0
    z = X @ W.t()
    z[:, mask] = float("-inf")
    dz = torch.softmax(z, 1)
    dz.scatter_add_(1, torch.where(live, y, 0)[:, None], -torch.ones_like(z[:, :1]))
    return dz * (dloss.double() * live)[:, None], X, W


@pytest.mark.parametrize("T,dtype", [(t, BF16) for t in (1, 40, 64, 128, 300, (1 << 18) + 100)] + [(t, F32) for t in (5, 40, 300)])
@pytest.mark.parametrize("padding", [0.0, 0.3, 1.0])
def test_masked_tokens_get_no_gradient(T, dtype, padding):
    """dZ of a masked token is 0 in every row, so its weights' gradient is 0: rows of padding, the caller's and the kernels' own, must
    not make it 0 times an infinity.  The others follow the formula: dZ is rounded once, the output once, and 2^-12 is far above
    what fp32 logits of 64 terms and sums of T of them add (2^18 tokens of bf16: 2^14 steps of 21/16 2^-22)."""
    x, w, y, dloss = _inputs(T, dtype, padding)
    _, lse = dtp.linear_cross_entropy(x, w, y)
    dx, dw = dtp.linear_cross_entropy_backward(dloss, x, w, y, lse, check=True)
    dz, X, W = _reference(x, w, y, dloss)
    masked = torch.isinf(w[:, 0])
    assert (dw[masked] == 0).all()
    half = torch.finfo(dtype).eps / 2
    off = 1.01 * half + 2.0 ** -12 + (2.0 ** 14 * 21 / 16 * 2.0 ** -22 if T > 1 << 18 else 0.0)
    ref = dz.t() @ X
    assert ((dw.double() - ref).abs() <= half * ref.abs() + off * dz.abs().t() @ X.abs() + 1e-38).all()
    ref = dz @ W
    live = y != IGNORE
    # column 0 is 0 times an infinity in the formula too
    assert ((dx.double() - ref).abs() <= half * ref.abs() + off * dz.abs() @ W.abs() + 1e-38)[live][:, 1:].all()


@pytest.mark.parametrize("T,dtype", [(t, BF16) for t in (2, 40, 300, (1 << 18) + 100)] + [(t, F32) for t in (2, 5, 32, 40, 300)])
@pytest.mark.parametrize("value", [float("-inf"), float("inf"), float("nan")])
def test_tokens_that_do_not_count_have_zero_rows(T, dtype, value):
    """Whatever stands in the weights: the gradient of a token without a target is 0, and not 0 times what is there."""
    x, w, y, dloss = _inputs(T, dtype, 0.5)
    y[0], y[1] = IGNORE, 7
    w[3, 5] = value
    _, lse = dtp.linear_cross_entropy(x, w, y)
    dx, _ = dtp.linear_cross_entropy_backward(dloss, x, w, y, lse)
    assert (dx[y == IGNORE] == 0).all()
