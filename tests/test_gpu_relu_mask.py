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


@pytest.mark.parametrize("T,K,N", [(1, 1025, 1), (1, 777, 40), (2, 2049, 333), (33, 1025, 200), (40, 1001, 17), (200, 2049, 300),
                                   (600, 1032, 136), (1100, 505, 130)])
def test_gate_of_the_block(T, K, N):
    """The mask of the block's gate, read off its gradient: a one in a column of its own for every token makes dW_gate's column
    that token's dG, which is dH U where the gate's sum is positive and zero elsewhere."""
    X, W_gate, z = _cancelling(T, K, N, seed=17)
    X = torch.cat([X, torch.eye(T, device=DEV, dtype=BF16)], 1).contiguous()
    W_gate = torch.cat([W_gate, torch.zeros((N, T), device=DEV, dtype=BF16)], 1).contiguous()
    W_up = torch.zeros_like(W_gate)
    W_up[:, K - 1] = 1.0
    W_down = torch.ones((K + T, N), device=DEV, dtype=BF16)
    Y, saved = dtp.gated_ffn(X, W_gate, W_up, W_down, activation="relu", save=True)
    _, dW_gate, _, _ = dtp.gated_ffn_backward(torch.ones_like(Y), X, W_gate, W_up, W_down, saved, activation="relu")
    assert torch.equal(dW_gate[:, K:].t().double(), torch.where(z > 0, float(K + T), 0.0).to(BF16).double())


@pytest.mark.parametrize("T,d,N", [(1, 64, 128), (2, 72, 200), (3, 520, 1001), (40, 136, 200), (300, 520, 333), (1000, 256, 640)])
def test_block_with_relu(T, d, N):
    """Value and gradients against the formulas in 64 bits; an element is off by at most its own rounding (2^-8) and, with the
    rounded factors H, dG and dU, 1.1 2^-8 of its terms' sizes."""
    def rand(seed, *shape, std=1.0):
        return (torch.randn(shape, generator=_gen(seed), device=DEV) * std).to(BF16)

    X, dY = rand(1, T, d), rand(2, T, d)
    Wg, Wu, Wd = rand(3, N, d, std=d ** -0.5), rand(4, N, d, std=d ** -0.5), rand(5, d, N, std=N ** -0.5)
    Y, saved = dtp.gated_ffn(X, Wg, Wu, Wd, activation="relu", save=True)
    got = (Y, *dtp.gated_ffn_backward(dY, X, Wg, Wu, Wd, saved, activation="relu"))
    x, wg, wu, wd, dy = (t.double() for t in (X, Wg, Wu, Wd, dY))
    g, u, dh = x @ wg.t(), x @ wu.t(), dy @ wd
    h, du, dg = g.clamp(min=0) * u, dh * g.clamp(min=0), dh * u * (g > 0)
    ref = (h @ wd.t(), dg @ wg + du @ wu, dg.t() @ x, du.t() @ x, dy.t() @ h)
    a = [t.abs() for t in (x, wg, wu, wd, h, dg, du, dy)]
    size = (a[4] @ a[3].t(), a[5] @ a[1] + a[6] @ a[2], a[5].t() @ a[0], a[6].t() @ a[0], a[7].t() @ a[4])
    for name, v, r, s in zip(("Y", "dX", "dW_gate", "dW_up", "dW_down"), got, ref, size):
        assert ((v.double() - r).abs() <= 2.0 ** -8 * (r.abs() + 1.1 * s)).all(), name
