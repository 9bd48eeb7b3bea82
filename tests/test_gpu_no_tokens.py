"""The backward passes without tokens: no input is read (NULL is allowed at the C ABI), the weights' gradients are zero."""
import pytest
import torch

from paper_2609_13846_gb300 import dtp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SIZES = pytest.mark.parametrize("d,N", [(64, 96), (65, 96), (64, 97), (9, 3), (1, 1)])
TYPES = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])


def _code(dtype):
    return dtp.DTP_BF16 if dtype is torch.bfloat16 else dtp.DTP_F32


@TYPES
@SIZES
def test_gated_backward(d, N, dtype):
    X = torch.empty((0, d), device=DEV, dtype=dtype)
    Wg, Wu, Wd = (torch.ones(s, device=DEV, dtype=dtype) for s in ((N, d), (N, d), (d, N)))
    Y, saved = dtp.gated_ffn(X, Wg, Wu, Wd, save=True)
    dX, *grads = dtp.gated_ffn_backward(Y, X, Wg, Wu, Wd, saved)
    assert dX.shape == (0, d) and all((g == 0).all() for g in grads)


@TYPES
@SIZES
@pytest.mark.parametrize("wanted", [(0, 1, 2), (0,), (2,), ()])
def test_gated_backward_without_inputs(d, N, dtype, wanted):
    out = [torch.full(s, 7.0, device=DEV, dtype=dtype) for s in ((N, d), (N, d), (d, N))]
    ws = dtp.gated_ffn_workspace(0, d, N, dtype, DEV, backward=True)
    st = dtp.lib().dtp_gated_ffn_backward(*[None] * 7, 0, d, N, dtp.ACTIVATIONS["silu"], _code(dtype), None,
                                          *(t.data_ptr() if i in wanted else None for i, t in enumerate(out)), ws.data_ptr(),
                                          ws.numel(), torch.cuda.current_stream().cuda_stream)
    assert st == dtp.DTP_OK and dtp.workspace_status(ws) == dtp.DTP_OK
    assert all((t == (0 if i in wanted else 7)).all() for i, t in enumerate(out))


@TYPES
@SIZES
def test_linear_backward_without_inputs(d, N, dtype):
    dW, db = torch.full((N, d), 7.0, device=DEV, dtype=dtype), torch.full((N,), 7.0, device=DEV, dtype=dtype)
    ws = dtp.linear_workspace(0, d, N, dtype, DEV, backward=True)
    st = dtp.lib().dtp_linear_backward(*[None] * 4, 0, d, N, dtp.ACTIVATIONS["gelu"], _code(dtype), None, dW.data_ptr(),
                                       db.data_ptr(), ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
    assert st == dtp.DTP_OK and dtp.workspace_status(ws) == dtp.DTP_OK
    assert (dW == 0).all() and (db == 0).all()
