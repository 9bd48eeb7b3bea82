"""Softmax cross entropy over a vocabulary and its gradients against the formulas in fp64."""
import pytest
import torch

from paper_2609_13846_gb300 import dtp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
IGNORE = -100


def _inputs(T, d, V, dtype, seed=0, scale=2.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn((T, d), generator=g, device=DEV).to(dtype)
    w = (torch.randn((V, d), generator=g, device=DEV) * scale / d ** 0.5).to(dtype)
    y = torch.randint(0, V, (T,), generator=g, device=DEV)
    y[torch.rand(T, generator=g, device=DEV) < 0.2] = IGNORE
    dloss = torch.rand(T, generator=g, device=DEV) / T
    return x, w, y, dloss


def _check(x, w, y, dloss, loss, lse, dx=None, dw=None, ignore=IGNORE):
    """Bounds: a logit is a sum of d products that the tensor cores cut off at 21/16 2^-22 of the terms' sizes for every 16
    (fp32: 2^-24 for every term); lse takes that of the worst logit and 2^-14 for its own sum (1024 roundings on any path to it)
    and rounding; a probability takes both; dZ is rounded once, and the gradients' sums of V or T terms are cut off alike."""
    bf16 = x.dtype == torch.bfloat16
    X, W = x.double(), w.double()
    T, d = X.shape
    V = W.shape[0]

    def sums(k):
        return (k / 16 + 4) * 21 / 16 * 2.0 ** -22 if bf16 else (k + 4) * 2.0 ** -24

    z = X @ W.t()
    zerr = sums(d) * (X.abs() @ W.abs().t()).amax(1)
    L = torch.logsumexp(z, 1)
    lerr = zerr + 2.0 ** -14 + 2.0 ** -22 * L.abs()
    live = y != ignore
    at = torch.where(live, y, torch.zeros_like(y))[:, None]
    assert ((lse.double() - L).abs() <= lerr).all()
    want = torch.where(live, L - z.gather(1, at)[:, 0], torch.zeros_like(L))
    assert ((loss.double() - want).abs() <= lerr + zerr).all()
    assert (loss[~live] == 0).all()
    if dx is None:
        return
    p = torch.exp(z - L[:, None])
    hit = torch.zeros_like(z).scatter_(1, at, 1.0)
    g = torch.where(live, dloss.double(), torch.zeros_like(L))[:, None]
    half = torch.finfo(x.dtype).eps / 2
    dz = (p - hit) * g
    # a probability's error, the difference's rounding, and the rounding of dZ
    off = ((2 * lerr[:, None] + 2.0 ** -20) * p + 2.0 ** -23 * hit) * g.abs() + 1.01 * half * dz.abs()
    for got, a, b, e, k in ((dx, dz, W, off, V), (dw, dz.t(), X, off.t(), T)):
        ref = a @ b
        assert ((got.double() - ref).abs() <= half * ref.abs() + (e + 2 * sums(k) * a.abs()) @ b.abs() + 1e-38).all()
    assert (dx[~live] == 0).all()


# fp32 has kernels of its own up to 32 tokens, with X whole in shared memory or in pieces
FEW = [(1, 1000, 33), (8, 130, 4096), (9, 2, 70), (16, 1537, 520), (17, 12, 999), (25, 2048, 321), (31, 3, 64), (32, 768, 1000),
       (32, 1600, 97), (33, 40, 515)]
SIZES = FEW + [(1, 1, 1), (1, 8, 2), (1, 64, 1000), (2, 72, 129), (3, 40, 8193), (7, 100, 257), (17, 256, 5003), (64, 136, 640),
         (65, 136, 641), (100, 64, 128), (128, 512, 1024), (129, 65, 1023), (257, 520, 5003), (300, 1024, 2500), (515, 96, 40001),
         (1000, 64, 300), (2048, 128, 70)]


@pytest.mark.parametrize("T,d,V", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_formula(T, d, V, dtype):
    x, w, y, dloss = _inputs(T, d, V, dtype)
    loss, lse = dtp.linear_cross_entropy(x, w, y, check=True)
    dx, dw = dtp.linear_cross_entropy_backward(dloss, x, w, y, lse, check=True)
    _check(x, w, y, dloss, loss, lse, dx, dw)


@pytest.mark.parametrize("T,d,V", [(20000, 64, 40000), (4096, 256, 131072)])
def test_several_pieces(T, d, V):
    """Logits that do not fit a piece, forward and backward; tokens drawn for the check."""
    x, w, y, dloss = _inputs(T, d, V, torch.bfloat16)
    loss, lse = dtp.linear_cross_entropy(x, w, y)
    some = torch.arange(0, T, 331, device=DEV)
    _check(x[some], w, y[some], dloss[some], loss[some], lse[some])
    # tokens without a gradient leave the others' sums to check
    quiet = torch.zeros_like(dloss)
    quiet[some] = dloss[some]
    dx, dw = dtp.linear_cross_entropy_backward(quiet, x, w, y, lse)
    _check(x[some], w, y[some], quiet[some], loss[some], lse[some], dx[some], dw)
    assert (dx[(quiet == 0)] == 0).all()


@pytest.mark.parametrize("T", [3, 70, 300])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_padding_and_targets_out_of_range(T, dtype):
    """Rows of padding may hold anything; targets that are no token's are reported and touch nothing else."""
    x, w, y, dloss = _inputs(T, 80, 300, dtype)
    y[0], y[1], y[2] = IGNORE, 5, 7
    clean, wanted = x.clone(), dloss.clone()
    for value in (float("nan"), float("inf")):
        x[0], dloss[0] = value, value
        loss, lse = dtp.linear_cross_entropy(x, w, y, check=True)
        dx, dw = dtp.linear_cross_entropy_backward(dloss, x, w, y, lse, check=True)
        live = slice(1, T)
        _check(clean[live], w, y[live], wanted[live], loss[live], lse[live], dx[live], dw)
        assert loss[0] == 0 and (dx[0] == 0).all()
    for bad in (300, -1, 1 << 40, -(1 << 63)):
        y2 = y.clone()
        y2[0] = bad
        ws = dtp.linear_cross_entropy_workspace(T, 80, 300, dtype, DEV, backward=True)
        loss, lse = dtp.linear_cross_entropy(clean, w, y2, workspace=ws)
        assert dtp.workspace_status(ws) == dtp.DTP_ERR_ARG
        assert torch.isnan(loss[0])
        dx, dw = dtp.linear_cross_entropy_backward(wanted, clean, w, y2, lse, workspace=ws)
        assert dtp.workspace_status(ws) == dtp.DTP_ERR_ARG
        y2[0] = IGNORE
        loss[0] = 0
        _check(clean, w, y2, wanted, loss, lse, dx, dw)
        dtp.linear_cross_entropy(clean, w, y2, workspace=ws)       # a good call clears the status
        assert dtp.workspace_status(ws) == dtp.DTP_OK
    # any value may mark the padding, a token's id too
    y3 = torch.where(y == IGNORE, torch.full_like(y, 9), y)
    loss, lse = dtp.linear_cross_entropy(clean, w, y3, ignore_index=9, check=True)
    dx, dw = dtp.linear_cross_entropy_backward(wanted, clean, w, y3, lse, ignore_index=9, check=True)
    _check(clean, w, y3, wanted, loss, lse, dx, dw, ignore=9)


@pytest.mark.parametrize("T", [2, 130])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_all_padding_and_no_tokens(T, dtype):
    x, w, y, dloss = _inputs(T, 64, 200, dtype)
    y[:] = IGNORE
    loss, lse = dtp.linear_cross_entropy(x, w, y, check=True)
    dx, dw = dtp.linear_cross_entropy_backward(dloss, x, w, y, lse, check=True)
    assert (loss == 0).all() and (dx == 0).all() and (dw == 0).all()
    loss, lse = dtp.linear_cross_entropy(x[:0], w, y[:0], check=True)
    dx, dw = dtp.linear_cross_entropy_backward(dloss[:0], x[:0], w, y[:0], lse, check=True)
    assert loss.shape == (0,) and dx.shape == (0, 64) and (dw == 0).all()


@pytest.mark.parametrize("T", [4, 200])
def test_large_logits(T):
    """Logits of thousands: exponentials far below and above fp32's range; one token far ahead of the others."""
    x, w, y, dloss = _inputs(T, 64, 1000, torch.bfloat16, scale=1000.0)
    loss, lse = dtp.linear_cross_entropy(x, w, y)
    dx, dw = dtp.linear_cross_entropy_backward(dloss, x, w, y, lse)
    assert all(torch.isfinite(t).all() for t in (loss, lse, dx, dw))
    X, W = x.double(), w.double()
    z = X @ W.t()
    L = torch.logsumexp(z, 1)
    zerr = 8 * 21 / 16 * 2.0 ** -22 * (X.abs() @ W.abs().t()).amax(1)
    assert ((lse.double() - L).abs() <= zerr + 2.0 ** -14 + 2.0 ** -22 * L.abs()).all()


def test_offsets_of_the_vectors():
    """Targets and vectors over tokens are often shifted by one: views on 8 and 4 byte boundaries."""
    x, w, y, dloss = _inputs(100, 64, 500, torch.bfloat16)
    tokens = torch.cat([y[:1], y])
    big = torch.zeros(101, device=DEV)
    big[1:] = dloss
    loss, lse = dtp.linear_cross_entropy(x, w, tokens[1:])
    lbig = torch.cat([lse[:1], lse])
    dx, dw = dtp.linear_cross_entropy_backward(big[1:], x, w, tokens[1:], lbig[1:])
    _check(x, w, y, dloss, loss, lse, dx, dw)


def test_gradient_against_differences():
    """fp64 central differences of the formula along a direction; the third derivatives of these logits are of order one, so
    the differences are good to 1e-6 of the slope's terms."""
    x, w, y, dloss = _inputs(9, 24, 50, torch.float32)
    _, lse = dtp.linear_cross_entropy(x, w, y)
    dx, dw = dtp.linear_cross_entropy_backward(dloss, x, w, y, lse)
    live = y != IGNORE

    def value(x, w):
        z = x @ w.t()
        per = torch.logsumexp(z, 1) - z.gather(1, torch.where(live, y, 0)[:, None])[:, 0]
        return (per * dloss.double())[live].sum()

    g = torch.Generator(device=DEV).manual_seed(3)
    for wx, ww in ((1.0, 0.0), (0.0, 1.0)):
        ax = wx * torch.randn(x.shape, generator=g, device=DEV, dtype=torch.float64)
        aw = ww * torch.randn(w.shape, generator=g, device=DEV, dtype=torch.float64)
        h = 1e-4
        diff = (value(x.double() + h * ax, w.double() + h * aw) - value(x.double() - h * ax, w.double() - h * aw)) / (2 * h)
        got = (dx.double() * ax).sum() + (dw.double() * aw).sum()
        size = (dx.double() * ax).abs().sum() + (dw.double() * aw).abs().sum()
        assert abs(got - diff) <= 1e-5 * size


@pytest.mark.parametrize("T,d,V", [(5, 64, 700), (300, 72, 3001)])
def test_repeats_streams_and_graphs(T, d, V):
    x, w, y, dloss = _inputs(T, d, V, torch.bfloat16)

    def both(stream=None, ws=None):
        loss, lse = dtp.linear_cross_entropy(x, w, y, stream=stream, workspace=ws)
        return (loss, lse, *dtp.linear_cross_entropy_backward(dloss, x, w, y, lse, stream=stream, workspace=ws))

    first = both()
    assert all(torch.equal(a, b) for a, b in zip(first, both()))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    second = both(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    ws = dtp.linear_cross_entropy_workspace(T, d, V, torch.bfloat16, DEV, backward=True)
    graphs = []
    for _ in range(2):                      # two graphs that share a workspace, one after the other
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = both(ws=ws)
        graphs.append((graph, out))
    for graph, out in graphs + graphs:
        ws.fill_(255)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(first, out))


@pytest.mark.parametrize("T,d,V,dtype", [(17000, 64, 131072, torch.bfloat16), (16500, 24, 300, torch.float32)])
def test_several_runs_of_tokens(T, d, V, dtype):
    """More tokens than the forward pass takes at once: the runs meet at their edges."""
    x, w, y, dloss = _inputs(T, d, V, dtype)
    loss, lse = dtp.linear_cross_entropy(x, w, y, check=True)
    some = torch.cat([torch.arange(0, T, 97, device=DEV), torch.arange(16384 - 3, 16384 + 3, device=DEV), torch.tensor([T - 1], device=DEV)])
    _check(x[some], w, y[some], dloss[some], loss[some], lse[some])


def test_very_many_tokens():
    """More than 2^18: dW is made in runs, whose sums are added in 64 bits."""
    T, d, V = (1 << 18) + 100, 64, 300
    x, w, y, dloss = _inputs(T, d, V, torch.bfloat16)
    loss, lse = dtp.linear_cross_entropy(x, w, y, check=True)
    dx, dw = dtp.linear_cross_entropy_backward(dloss, x, w, y, lse, check=True)
    some = torch.arange(0, T, 1009, device=DEV)
    X, W = x.double(), w.double()
    live = (y != IGNORE).double()
    g = (dloss.double() * live)[:, None]
    dz = torch.softmax(X @ W.t(), 1)
    dz.scatter_add_(1, torch.where(y == IGNORE, 0, y)[:, None], -torch.ones_like(g))
    dz *= g
    half = torch.finfo(torch.bfloat16).eps / 2
    # dZ's rounding and a probability's error (2^-13), the runs' sums (2^18 terms in 2^14 steps of 21/16 2^-22), the output's rounding
    off = (1.01 * half + 2.0 ** -13 + 2.0 ** 14 * 21 / 16 * 2.0 ** -22) * dz.abs()
    ref = dz.t() @ X
    assert ((dw.double() - ref).abs() <= half * ref.abs() + off.t() @ X.abs()).all()
    ref = dz[some] @ W
    assert ((dx[some].double() - ref).abs() <= half * ref.abs() + off[some] @ W.abs()).all()


@pytest.mark.parametrize("T,dtype", [(5, torch.bfloat16), (100, torch.bfloat16), (5, torch.float32), (100, torch.float32)])
def test_one_gradient_alone(T, dtype):
    """At the C ABI either gradient may be left out."""
    x, w, y, dloss = _inputs(T, 72, 900, dtype)
    _, lse = dtp.linear_cross_entropy(x, w, y)
    dx, dw = dtp.linear_cross_entropy_backward(dloss, x, w, y, lse)
    ws = dtp.linear_cross_entropy_workspace(T, 72, 900, dtype, DEV, backward=True)
    for one in (True, False):
        a, b = torch.full_like(x, 7.0), torch.full_like(w, 7.0)
        st = dtp.lib().dtp_linear_cross_entropy_backward(
            dloss.data_ptr(), x.data_ptr(), w.data_ptr(), y.data_ptr(), lse.data_ptr(), T, 72, 900, IGNORE, dtp._torch_code(dtype),
            a.data_ptr() if one else None, None if one else b.data_ptr(), ws.data_ptr(), ws.numel(),
            torch.cuda.current_stream().cuda_stream)
        assert st == dtp.DTP_OK
        assert torch.equal(a, dx if one else torch.full_like(x, 7.0)) and torch.equal(b, torch.full_like(w, 7.0) if one else dw)


@pytest.mark.parametrize("scale", [1e-30, 1.0, 1e30])
def test_gradients_of_any_size(scale):
    """dloss far from one, and of both signs: dZ is held in units of its largest size."""
    x, w, y, dloss = _inputs(150, 64, 400, torch.bfloat16)
    dloss = dloss * 150 * scale
    dloss[::3] *= -1e-4
    loss, lse = dtp.linear_cross_entropy(x, w, y)
    dx, dw = dtp.linear_cross_entropy_backward(dloss, x, w, y, lse)
    _check(x, w, y, dloss, loss, lse, dx, dw)
    dx, dw = dtp.linear_cross_entropy_backward(torch.zeros_like(dloss), x, w, y, lse)
    assert (dx == 0).all() and (dw == 0).all()


@pytest.mark.parametrize("T,dtype", [(40, torch.bfloat16), (300, torch.bfloat16), (20, torch.float32), (70, torch.float32)])
def test_infinite_logits(T, dtype):
    """A logit of infinity: lse and the other tokens' loss are infinite, its own loss is no number; a vocabulary of -inf but for
    one token has that token's logit as lse; a NaN stays in its row."""
    x, w, y, _ = _inputs(T, 64, 500, dtype)
    x = x.abs()
    x[3, 5] = float("nan")
    y[:] = 7
    y[0] = 100
    w[100] = w[100].abs() + 0.1
    w[100, 0] = float("inf")
    x[:, 0] = 1.0
    loss, lse = dtp.linear_cross_entropy(x, w, y)
    others = torch.ones(T, dtype=torch.bool, device=DEV)
    others[3] = False
    assert torch.isinf(lse[others]).all() and (lse[others] > 0).all() and torch.isnan(lse[3])
    assert torch.isnan(loss[0]) and torch.isinf(loss[1]) and torch.isnan(loss[3])
    w[:, 0] = float("-inf")
    w[7, 0] = 0.0
    loss, lse = dtp.linear_cross_entropy(x, w, y)
    z = (x.double() * w[7].double()).sum(1)
    far = others.clone()
    far[0] = False
    assert ((lse[far].double() - z[far]).abs() <= 1e-4).all() and (loss[far].abs() <= 1e-4).all() and torch.isinf(loss[0])


def test_weights_beyond_32_bits():
    """A vocabulary whose weights have more than 2^31 elements: its last tokens are read, and written, where they are."""
    T, d, V = 70, 2304, 1 << 20
    g = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn((T, d), generator=g, device=DEV).to(torch.bfloat16)
    w = torch.empty((V, d), dtype=torch.bfloat16, device=DEV)
    for v in range(0, V, 1 << 17):
        w[v:v + (1 << 17)] = torch.randn((1 << 17, d), generator=g, device=DEV) / 48.0
    assert w.numel() > 1 << 31
    y = torch.randint(V - 1000, V, (T,), generator=g, device=DEV)
    z = torch.cat([x.double() @ w[v:v + (1 << 16)].double().t() for v in range(0, V, 1 << 16)], 1)
    L = torch.logsumexp(z, 1)
    loss, lse = dtp.linear_cross_entropy(x, w, y, check=True)
    assert ((lse.double() - L).abs() <= 1e-4).all()
    assert ((loss.double() - (L - z.gather(1, y[:, None])[:, 0])).abs() <= 2e-4).all()
    dloss = torch.full((T,), 1.0 / T, device=DEV)
    dx, dw = dtp.linear_cross_entropy_backward(dloss, x, w, y, lse, check=True)
    dz = torch.exp(z - L[:, None])
    dz.scatter_add_(1, y[:, None], -torch.ones_like(L)[:, None])
    dz /= T
    for rows in (slice(0, 1000), slice(V // 2 - 500, V // 2 + 500), slice(V - 1000, V)):
        ref = dz[:, rows].t() @ x.double()
        assert (dw[rows].double() - ref).norm() <= 4e-3 * ref.norm()
    ref = sum(dz[:, v:v + (1 << 16)] @ w[v:v + (1 << 16)].double() for v in range(0, V, 1 << 16))
    assert (dx.double() - ref).norm() <= 4e-3 * ref.norm()
