"""Weight gradients over very many tokens: sums of one sign, in which an accumulator that cuts its sums off loses the most.

Tolerances: the output's rounding (2^-8 bf16, 2^-24 fp32) and 2^-11 of the sum of the terms' sizes: 2^18 terms in one run cut off
at 2^-26 of the running sum for every 16 are 2^-12, fp32 sums of as many random roundings of 2^-24 less (2^-15)."""
import pytest
import torch

from paper_2609_13846_gb300 import dtp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _rand(seed, T, n, dtype):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (0.5 + 0.5 * torch.rand((T, n), generator=g, device=DEV)).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,K,N", [((1 << 18) + 1, 8, 24), ((1 << 19) + 77, 9, 5), ((1 << 26) - 3, 8, 8)])
def test_linear_weight_gradient(T, K, N, dtype):
    X, dY, W = _rand(1, T, K, dtype), _rand(2, T, N, dtype), _rand(3, N, K, dtype)
    dX, dW, db = dtp.linear_backward(dY, X, W, bias=True)
    ref = sum(dY[i:i + (1 << 22)].double().t() @ X[i:i + (1 << 22)].double() for i in range(0, T, 1 << 22))
    u = 2.0 ** -8 if dtype is torch.bfloat16 else 2.0 ** -24
    assert ((dW.double() - ref).abs() <= (u + 2.0 ** -11) * ref).all()
    again = dtp.linear_backward(dY, X, W, bias=True)
    assert torch.equal(dW, again[1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,d,N", [((1 << 18) + 5, 16, 9), ((1 << 23) + 1, 8, 8)])
def test_gated_weight_gradients(T, d, N, dtype):
    """All values are positive, and so are all terms; a tenth more than two roundings for the rounded factors."""
    X, dY = _rand(1, T, d, dtype), _rand(2, T, d, dtype)
    Wg, Wu, Wd = _rand(3, N, d, dtype), _rand(4, N, d, dtype), _rand(5, d, N, dtype)
    _, saved = dtp.gated_ffn(X, Wg, Wu, Wd, activation="none", save=True)
    grads = dtp.gated_ffn_backward(dY, X, Wg, Wu, Wd, saved, activation="none")
    ref = [0.0, 0.0, 0.0]
    for i in range(0, T, 1 << 21):
        x, dy = X[i:i + (1 << 21)].double(), dY[i:i + (1 << 21)].double()
        g, u, dh = x @ Wg.double().t(), x @ Wu.double().t(), dy @ Wd.double()
        for j, a in enumerate(((dh * u).t() @ x, (dh * g).t() @ x, dy.t() @ (g * u))):
            ref[j] = ref[j] + a
    u = 2.1 * 2.0 ** -8 if dtype is torch.bfloat16 else 2.0 ** -22
    for got, want in zip(grads[1:], ref):
        assert ((got.double() - want).abs() <= (u + 2.0 ** -11) * want).all()


def test_the_most_tokens():
    """2^31 - 256 tokens of ones: every sum is that number, far beyond what one fp32 accumulator can count."""
    T, K, N = (1 << 31) - 256, 8, 8
    torch.cuda.empty_cache()
    X = torch.ones((T, K), device=DEV, dtype=torch.bfloat16)
    dW = torch.zeros((N, K), device=DEV, dtype=torch.bfloat16)
    db = torch.zeros((N,), device=DEV, dtype=torch.bfloat16)
    ws = dtp.linear_workspace(T, K, N, torch.bfloat16, DEV, backward=True)
    st = dtp.lib().dtp_linear_backward(X.data_ptr(), X.data_ptr(), None, None, T, K, N, 0, dtp.DTP_BF16, None, dW.data_ptr(),
                                       db.data_ptr(), ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
    assert st == dtp.DTP_OK and dtp.workspace_status(ws) == dtp.DTP_OK
    assert (dW == 2.0 ** 31).all() and (db == 2.0 ** 31).all()
    del X, ws
    torch.cuda.empty_cache()
