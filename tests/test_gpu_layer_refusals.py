"""Workspaces that the layer operators refuse before the library sees them."""
import pytest
import torch

from paper_2609_13846_gb300 import dtp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

BAD = [lambda n: torch.empty(n, dtype=torch.uint8),                                     # on the host
       lambda n: torch.empty(1, dtype=torch.uint8, device=DEV).expand(n),               # many elements of one byte
       lambda n: torch.empty(2 * n, dtype=torch.uint8, device=DEV)[::2],
       lambda n: torch.empty(n, dtype=torch.float32, device=DEV)]


@pytest.mark.parametrize("bad", BAD, ids=["host", "expanded", "strided", "f32"])
def test_workspace(bad):
    ws = bad(1 << 20)
    X, W = torch.ones((4, 8), device=DEV), torch.ones((16, 8), device=DEV)
    with pytest.raises(ValueError, match="workspace"):
        dtp.linear(X, W, workspace=ws)
    with pytest.raises(ValueError, match="workspace"):
        dtp.linear_backward(torch.ones((4, 16), device=DEV), X, W, workspace=ws)
    Y, saved = dtp.gated_ffn(X, W, W, W.t().contiguous(), save=True)
    with pytest.raises(ValueError, match="workspace"):
        dtp.gated_ffn(X, W, W, W.t().contiguous(), workspace=ws)
    with pytest.raises(ValueError, match="workspace"):
        dtp.gated_ffn_backward(Y, X, W, W, W.t().contiguous(), saved, workspace=ws)
    with pytest.raises(ValueError, match="workspace"):
        dtp.clip_grad_norm([X], 1.0, workspace=ws)
