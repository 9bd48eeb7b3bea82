"""The signs of the saved pre-activations that relu's gradient goes by, where sums cancel.

The terms come in pairs that cancel exactly, in an order that lets the running sum grow first, and one more term decides: the
exact sum is that term (or zero), some 2^-37 of the sum of the terms' sizes.  All products are multiples of 2^-24 and all
sums below 2^15, so sums in 64 bits are exact in any order."""
import pytest
import torch

from paper_2609_13846_gb300 import dtp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _cancelling(T, K, N, seed=0):
    """(X [T, K], W [N, K], the exact sums): columns 0 .. h - 1 and h .. 2h - 1 cancel, the last one decides."""
    h = (K - 1) // 2
    u = torch.randint(1, 200, (T, h), generator=_gen(seed), device=DEV) / 64.0
    v = torch.randint(1, 200, (N, h), generator=_gen(seed + 1), device=DEV) / 64.0
    sign = torch.randint(-1, 2, (N,), generator=_gen(seed + 2), device=DEV).double()
    X = torch.zeros((T, K), device=DEV)
    W = torch.zeros((N, K), device=DEV)
    X[:, :h], X[:, h:2 * h], X[:, -1] = u, u, 1.0
    W[:, :h], W[:, h:2 * h], W[:, -1] = v, -v, sign * 2.0 ** -24
    return X.to(BF16), W.to(BF16), (sign * 2.0 ** -24).expand(T, N)


SIZES = [(1, 1025, 1), (1, 4097, 40), (2, 777, 333), (5, 2049, 1), (40, 2049, 200), (70, 1001, 3), (200, 4104, 300),
         (600, 1032, 264), (1500, 2049, 130)]


@pytest.mark.parametrize("T,K,N", SIZES)
def test_cancelling_sums(T, K, N):
    X, W, z = _cancelling(T, K, N)
    _, Z = dtp.linear(X, W, activation="relu", save=True)
    assert torch.equal(torch.sign(Z.double()), torch.sign(z))


@pytest.mark.parametrize("T", [1, 2, 40, 300])
def test_a_bias_that_cancels(T):
    """Sums of one size that the bias takes away but for a last term: no large value is near."""
    K, N = 2048, 130
    X, W, z = _cancelling(T, K, N, seed=5)
    W[:, 0] += 64.0
    X[:, 0] = 2.0
    W[:, (K - 1) // 2] = -(W[:, 0] - 64.0)          # 2 W_0 - 2 (W_0 - 64) = 128 before the bias
    X[:, (K - 1) // 2] = 2.0
    b = torch.full((N,), -128.0, device=DEV, dtype=BF16)
    exact = X.double() @ W.double().t() + b.double()
    _, Z = dtp.linear(X, W, b, activation="relu", save=True)
    assert torch.equal(torch.sign(Z.double()), torch.sign(exact))


@pytest.mark.parametrize("T", [1, 20, 100, 700])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_a_sum_that_comes_out_as_zero(T, sign):
    """1 + s 2^-40 - 1 in sums of 24 bits is zero; exactly it has a sign."""
    X = torch.zeros((T, 192), device=DEV, dtype=BF16)
    W = torch.zeros((96, 192), device=DEV, dtype=BF16)
    X[:, 0], X[:, 64], X[:, 128] = 1.0, 2.0 ** -20, 1.0
    W[:, 0], W[:, 64], W[:, 128] = 1.0, sign * 2.0 ** -20, -1.0
    Y, Z = dtp.linear(X, W, activation="relu", save=True)
    assert (torch.sign(Z) == sign).all()
    dX, _, _ = dtp.linear_backward(torch.ones_like(Y), X, W, Z, activation="relu")
    assert ((dX[:, 0] != 0) == (sign > 0)).all()


@pytest.mark.parametrize("T", [1, 33, 500])
def test_empty_rows_and_infinities(T):
    """Rows of zeros give zeros; infinities and NaN stay in their rows and columns."""
    X, W, z = _cancelling(T, 1025, 60, seed=8)
    X[0] = 0
    W[7] = 0
    _, Z = dtp.linear(X, W, activation="relu", save=True)
    assert (Z[0] == 0).all() and (Z[:, 7] == 0).all()
    keep = torch.ones_like(Z, dtype=torch.bool)
    keep[0], keep[:, 7] = False, False
    assert torch.equal(torch.sign(Z.double())[keep], torch.sign(z)[keep])
    X[0, 5], W[9, 3] = float("inf"), float("nan")
    _, Z2 = dtp.linear(X, W, activation="relu", save=True)
    keep[:, 9] = False
    assert torch.equal(Z2[keep], Z[keep]) and not torch.isfinite(Z2[0]).any() and torch.isnan(Z2[:, 9]).all()


@pytest.mark.parametrize("scale", [2.0 ** -50, 2.0 ** 50])
def test_scales_whose_products_leave_fp32s_squares(scale):
    """Rows whose squared norms vanish or overflow in fp32."""
    X, W, z = _cancelling(300, 1025, 64, seed=11)
    _, Z = dtp.linear((X.float() * scale * scale).to(BF16), (W.float() / scale).to(BF16), activation="relu", save=True)
    assert torch.equal(torch.sign(Z.double()), torch.sign(z))


@pytest.mark.parametrize("T,N", [(1, 1), (1, 130), (3, 129), (5, 31), (66, 1)])
def test_nothing_beyond_the_rows_is_touched(T, N):
    """Pieces of the last rows and columns are whole; what lies beyond them in memory keeps its bits."""
    K = 192
    X, W, z = _cancelling(T, K, N, seed=13)
    b = torch.ones(N, device=DEV, dtype=BF16)
    ws = dtp.linear_workspace(T, K, N, BF16, DEV)
    store = torch.full((T * N + 4096,), 7.0, device=DEV)
    Y = torch.empty((T, N), device=DEV, dtype=BF16)
    st = dtp.lib().dtp_linear(X.data_ptr(), W.data_ptr(), b.data_ptr(), None, T, K, N, dtp.ACTIVATIONS["relu"], dtp.DTP_BF16,
                              Y.data_ptr(), store.data_ptr(), ws.data_ptr(), ws.numel(),
                              torch.cuda.current_stream().cuda_stream)
    assert st == dtp.DTP_OK and dtp.workspace_status(ws) == dtp.DTP_OK
    assert (store[T * N:] == 7).all() and (store[:T * N] > 0.9).all()
