"""The layer products at sizes that reach every tile form: many rounds, split tiles, left-over tiles, narrow tiles, both
operand orders with odd edges, offsets beyond 2^31.  Tolerances as in test_gpu_layers: an element is off by at most one bf16
rounding (2^-8) of itself and 2^-16 of the sum of its terms' sizes, plus 2^-8 of that sum where the terms were rounded."""
import math

import pytest
import torch

from paper_2609_13846_gb300 import dtp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16
U = 2.0 ** -8


def _rand(seed, *shape, std=1.0, dtype=BF16):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def _check(got, a, b, rounded, what):
    """got = a b^T with a [M,K], b [N,K] in fp64."""
    ref, terms = a @ b.t(), a.abs() @ b.abs().t()
    bound = U * ref.abs() + (1.1 * U if rounded else 2.0 ** -16) * terms
    d = (got.double() - ref).abs()
    assert (d <= bound).all(), (what, (d / bound).max().item())
    assert d.norm().item() <= 3e-3 * ref.norm().item(), what


# (T, K, N): one round of wide pairs; several rounds with left-over tiles split; few tiles with long sums; narrow
# tiles; one row beyond a tile; odd everything
PLAIN = [(2048, 256, 2048), (2560, 4096, 2048), (5000, 512, 2048), (300, 4096, 520), (256, 8192, 256), (129, 4096, 1000),
         (257, 2000, 136), (700, 64, 9000), (1500, 1001, 777), (90, 1024, 4104), (2000, 1024, 3080), (33, 4096, 9000)]


@pytest.mark.parametrize("T,K,N", PLAIN)
def test_linear_forward_and_both_gradients(T, K, N):
    X, W, dY = _rand(1, T, K), _rand(2, N, K, std=1 / math.sqrt(K)), _rand(3, T, N)
    Y = dtp.linear(X, W)
    dX, dW, db = dtp.linear_backward(dY, X, W, bias=True)
    x, w, dy = X.double(), W.double(), dY.double()
    _check(Y, x, w, False, "Y")
    _check(dX, dy, w.t(), False, "dX")
    _check(dW, dy.t(), x.t(), False, "dW")
    assert (db.double() - dy.sum(0)).abs().le(U * dy.sum(0).abs() + 2.0 ** -16 * dy.abs().sum(0)).all()
    assert torch.equal(Y, dtp.linear(X, W))
    again = dtp.linear_backward(dY, X, W, bias=True)
    assert all(torch.equal(a, b) for a, b in zip((dX, dW, db), again))


@pytest.mark.parametrize("T,K,N,act", [(2560, 1024, 2048, "silu"), (300, 2048, 264, "gelu"), (1000, 777, 1001, "silu"),
                                       (50, 2048, 9000, "gelu"), (4000, 64, 256, "relu")])
def test_full_epilogue(T, K, N, act):
    X, W, b, R = _rand(1, T, K), _rand(2, N, K, std=1 / math.sqrt(K)), _rand(3, N), _rand(4, T, N)
    Y, Z = dtp.linear(X, W, b, R, activation=act, save=True)
    z = X.double() @ W.double().t() + b.double()
    size = X.double().abs() @ W.double().t().abs() + b.double().abs()
    assert ((Z.double() - z).abs() <= 2.0 ** -16 * size).all()
    y = {"silu": lambda: z * torch.sigmoid(z), "gelu": lambda: z * torch.special.ndtr(z),
         "relu": lambda: z.clamp(min=0)}[act]() + R.double()
    assert ((Y.double() - y).abs() <= U * y.abs() + 2.0 ** -15 * (size + R.double().abs())).all()


@pytest.mark.parametrize("T,d,N", [(2600, 512, 1100), (200, 2048, 1024), (700, 128, 3000), (150, 4096, 264), (1300, 520, 333)])
def test_gated_block(T, d, N):
    X, Wg, Wu, Wd = (_rand(1, T, d), _rand(2, N, d, std=1 / math.sqrt(d)), _rand(3, N, d, std=1 / math.sqrt(d)),
                     _rand(4, d, N, std=1 / math.sqrt(N)))
    dY = _rand(5, T, d)
    Y, saved = dtp.gated_ffn(X, Wg, Wu, Wd, save=True)
    grads = dtp.gated_ffn_backward(dY, X, Wg, Wu, Wd, saved)
    x, wg, wu, wd, dy = (t.double() for t in (X, Wg, Wu, Wd, dY))
    g, u = x @ wg.t(), x @ wu.t()
    s = torch.sigmoid(g)
    h, dh = g * s * u, dy @ wd
    du, dg = dh * g * s, dh * u * s * (1 + g * (1 - s))
    _check(Y, h, wd, True, "Y")
    _check(grads[1], dg.t(), x.t(), True, "dW_gate")
    _check(grads[2], du.t(), x.t(), True, "dW_up")
    _check(grads[3], dy.t(), h.t(), True, "dW_down")
    _check(grads[0], torch.cat([dg, du], 1), torch.cat([wg, wu], 0).t(), True, "dX")


@pytest.mark.parametrize("N", [32768, 32767])
def test_offsets_beyond_two_to_the_31(N):
    """Y and Z of more than 2^31 elements: rows at the end are right and the ones before them untouched by overflow."""
    T, K = 70001, 16
    X, W, b = _rand(1, T, K), _rand(2, N, K, std=0.25), _rand(3, N)
    Y, Z = dtp.linear(X, W, b, activation="silu", save=True)
    for rows in (slice(0, 40), slice(65530, 65545), slice(T - 40, T)):
        z = X[rows].double() @ W.double().t() + b.double()
        size = X[rows].double().abs() @ W.double().t().abs() + b.double().abs()
        assert ((Z[rows].double() - z).abs() <= 2.0 ** -16 * size).all()
        y = z * torch.sigmoid(z)
        assert ((Y[rows].double() - y).abs() <= U * y.abs() + 2.0 ** -15 * size).all()
    dX, dW, _ = dtp.linear_backward(Y, X, W, Z, activation="silu")
    z = Z[T - 40:].double()
    s = torch.sigmoid(z)
    dz = Y[T - 40:].double() * s * (1 + z * (1 - s))
    _check(dX[T - 40:], dz, W.double().t(), True, "dX")


@pytest.mark.parametrize("T,K,N", [(2, 4096, 1000), (8, 5000, 333), (20, 1024, 777), (32, 8192, 64), (70, 3000, 1000)])
def test_f32_few_tokens_and_long_sums(T, K, N):
    X, W, b = _rand(1, T, K, dtype=torch.float32), _rand(2, N, K, dtype=torch.float32), _rand(3, N, dtype=torch.float32)
    Y = dtp.linear(X, W, b)
    ref = X.double() @ W.double().t() + b.double()
    terms = X.double().abs() @ W.double().t().abs() + b.double().abs()
    # K sequential additions at the very most: K 2^-24 of the terms; a hundredth of it is held (sqrt(K) and less in practice)
    assert ((Y.double() - ref).abs() <= max(4, K / 100) * 2.0 ** -24 * terms).all()


@pytest.mark.parametrize("T,K,N,bias", [(600, 4096, 520, True), (40, 2048, 1001, False), (1500, 777, 300, True), (2, 512, 999, True)])
def test_relu_mask_is_the_exact_signs(T, K, N, bias):
    """Saved pre-activations have the sign of the exact sum, outlier channels and all.  Left out is what the kernel's own
    compensated sums leave open: K / 32 additions of errors of 2^-24 of 2^-24 of the terms, below 2^-40 of them."""
    X, W = _rand(1, T, K), _rand(2, N, K, std=0.02)
    X[:, :4] *= 20
    b = _rand(3, N, std=0.5) if bias else None
    _, Z = dtp.linear(X, W, b, activation="relu", save=True)
    z = X.double() @ W.double().t() + (b.double() if bias else 0)
    size = X.double().abs() @ W.double().t().abs() + (b.double().abs() if bias else 0)
    clear = z.abs() > 2.0 ** -40 * size
    assert torch.equal((Z > 0) & clear, (z > 0) & clear)
    assert ((Z.double() - z).abs() <= 2.0 ** -16 * size).all()
