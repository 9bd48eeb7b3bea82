"""The linear layer and the gated feed-forward block, forward and backward, against the formulas in 64 bits.

Tolerances.  With u = 2^-8, the unit roundoff of bf16 (8 significant bits): an output is one rounding of a sum whose terms may carry
one rounding of their own (H, dG, dU, dZ), so an element is off by at most u |value| + u sum |terms|, or, where
the terms are not rounded, by u |value| and the fp32 sum's error, held to 2^-16 sum |terms| (sqrt(K) 2^-24 would be
2^-18 at K = 4096).  Ten per cent on the terms' share cover the fp32 errors of the factors.  Over an array of 4096
elements or more the roundings average: between u / sqrt(12) and u / sqrt(3) by the place within a binade, 1.7e-3
over all, for each of the two, 2.4e-3 in all, and a relative 2-norm of 3e-3 is held (for fewer elements the element
bound alone).  fp32: 2e-6
of the 2-norm, far below K 2^-24 (6e-5 at K = 1000) and well above sqrt(K) 2^-24; single elements eight times that
of the array's root mean square or of their own value.
"""
import math

import pytest
import torch

from paper_2609_13846_gb300 import dtp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -8
BF16, F32 = torch.bfloat16, torch.float32


def _rand(seed, *shape, dtype=BF16, std=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def _close(got, ref, what, terms=None, rounded=False):
    """got (bf16 or fp32) against ref (fp64), by the tolerances above; ``terms``: the sum of the terms' sizes."""
    d = got.double() - ref
    norm = ref.norm().item()
    assert torch.isfinite(got).all(), what
    if got.dtype is BF16:
        bound = U * ref.abs() + (1.1 * U if rounded else 2.0 ** -16) * terms
        assert (d.abs() <= bound + 1e-30).all(), (what, (d.abs() / bound).max().item())
        assert ref.numel() < 4096 or d.norm().item() <= 3e-3 * norm, (what, d.norm().item() / norm)
    else:
        assert d.norm().item() <= 2e-6 * norm + 1e-30, (what, d.norm().item() / max(norm, 1e-300))
        rms = norm / math.sqrt(max(1, ref.numel()))
        assert (d.abs() <= 1.6e-5 * torch.clamp(ref.abs(), min=rms) + 1e-30).all(), what


def _act(name, z):
    return {"none": lambda: z, "silu": lambda: z / (1 + torch.exp(-z)),
            "gelu": lambda: 0.5 * z * (1 + torch.erf(z / math.sqrt(2))), "relu": lambda: z.clamp(min=0)}[name]()


def _slope(name, z):
    s = 1 / (1 + torch.exp(-z))
    return {"none": lambda: torch.ones_like(z), "silu": lambda: s * (1 + z * (1 - s)),
            "gelu": lambda: 0.5 * (1 + torch.erf(z / math.sqrt(2))) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi),
            "relu": lambda: (z > 0).double()}[name]()


def _linear_case(T, K, N, act, bias, residual, dtype, seed=0, **kw):
    X, W = _rand(seed, T, K, dtype=dtype), _rand(seed + 1, N, K, dtype=dtype, std=1 / math.sqrt(K))
    b = _rand(seed + 2, N, dtype=dtype) if bias else None
    R = _rand(seed + 3, T, N, dtype=dtype) if residual else None
    dY = _rand(seed + 4, T, N, dtype=dtype)
    Y, Z = dtp.linear(X, W, b, R, activation=act, save=True, **kw)
    Y0 = dtp.linear(X, W, b, R, activation=act, **kw)
    dX, dW, db = dtp.linear_backward(dY, X, W, Z, activation=act, bias=bias)
    x, w, dy = X.double(), W.double(), dY.double()
    z = x @ w.t() + (b.double() if bias else 0)
    y = _act(act, z) + (R.double() if residual else 0)
    dz = dy * _slope(act, z)
    assert torch.equal(Y, Y0)
    size = x.abs() @ w.t().abs() + (b.double().abs() if bias else 0)
    _close(Y, y, "Y", 1.2 * size + (R.double().abs() if residual else 0))        # |act'| is below 1.13
    _close(Z, z, "Z")
    rounded = act != "none"
    _close(dX, dz @ w, "dX", dz.abs() @ w.abs(), rounded)
    _close(dW, dz.t() @ x, "dW", dz.t().abs() @ x.abs(), rounded)
    if bias:
        _close(db, dz.sum(0), "dbias", dz.abs().sum(0))
    else:
        assert db is None


SIZES = [(1, 64, 64), (1, 1, 1), (2, 7, 5), (3, 4096, 130), (17, 257, 129), (33, 40, 1000), (64, 520, 1001),
         (127, 128, 256), (128, 64, 128), (129, 72, 264), (200, 1000, 999), (257, 513, 300), (515, 96, 77),
         (1003, 256, 512)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,K,N", SIZES)
def test_linear_sizes(T, K, N, dtype):
    _linear_case(T, K, N, "silu", True, True, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 5, 150, 600])
@pytest.mark.parametrize("act", ["none", "silu", "gelu", "relu"])
@pytest.mark.parametrize("bias,residual", [(False, False), (True, False), (False, True)])
def test_linear_epilogues(T, act, bias, residual, dtype):
    if act == "relu":       # a kink: a pre-activation within rounding of zero may fall on either side
        X = torch.tensor([[1.0, -2.0], [3.0, 0.5]], device=DEV).to(dtype).repeat(T, 1)
        W = torch.tensor([[1.0, 1.0], [-1.0, 1.0], [2.0, 1.0]], device=DEV).to(dtype)
        Y, Z = dtp.linear(X, W, activation=act, save=True)
        z = X.double() @ W.double().t()
        assert torch.equal(Y.double(), z.clamp(min=0)) and torch.equal(Z.double(), z)
        dY = torch.ones_like(Y)
        dX, dW, _ = dtp.linear_backward(dY, X, W, Z, activation=act)
        dz = (z > 0).double()
        assert torch.equal(dX.double(), (dz @ W.double()).to(dtype).double())
        assert torch.equal(dW.double(), (dz.t() @ X.double()).to(dtype).double())
        return
    _linear_case(T, 136, 264, act, bias, residual, dtype, seed=10)


def _gated_ref(X, Wg, Wu, Wd, R, act, dY):
    """(value, sum of the terms' sizes) of Y, dX, dW_gate, dW_up and dW_down."""
    x, wg, wu, wd = (t.double() for t in (X, Wg, Wu, Wd))
    g, u = x @ wg.t(), x @ wu.t()
    h = _act(act, g) * u
    y = h @ wd.t() + (R.double() if R is not None else 0)
    dy = dY.double()
    dh = dy @ wd
    du, dg = dh * _act(act, g), dh * u * _slope(act, g)
    a = [t.abs() for t in (x, wg, wu, wd, h, dg, du, dy)]
    sizes = (a[4] @ a[3].t() + (R.double().abs() if R is not None else 0), a[5] @ a[1] + a[6] @ a[2], a[5].t() @ a[0],
             a[6].t() @ a[0], a[7].t() @ a[4])
    return list(zip((y, dg @ wg + du @ wu, dg.t() @ x, du.t() @ x, dy.t() @ h), sizes))


def _gated_inputs(T, d, N, dtype, seed=0):
    return (_rand(seed, T, d, dtype=dtype), _rand(seed + 1, N, d, dtype=dtype, std=1 / math.sqrt(d)),
            _rand(seed + 2, N, d, dtype=dtype, std=1 / math.sqrt(d)),
            _rand(seed + 3, d, N, dtype=dtype, std=1 / math.sqrt(N)))


GATED = [(1, 64, 128), (1, 1, 1), (2, 9, 3), (3, 520, 1001), (17, 96, 257), (32, 256, 512), (65, 136, 72),
         (128, 64, 128), (129, 65, 129), (250, 1000, 333), (257, 520, 640), (600, 128, 1000), (1030, 72, 264)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,d,N", GATED)
def test_gated_sizes(T, d, N, dtype):
    X, Wg, Wu, Wd = _gated_inputs(T, d, N, dtype)
    R, dY = _rand(8, T, d, dtype=dtype), _rand(9, T, d, dtype=dtype)
    Y, saved = dtp.gated_ffn(X, Wg, Wu, Wd, R, save=True)
    assert torch.equal(Y, dtp.gated_ffn(X, Wg, Wu, Wd, R))
    got = (Y, *dtp.gated_ffn_backward(dY, X, Wg, Wu, Wd, saved))
    ref = _gated_ref(X, Wg, Wu, Wd, R, "silu", dY)
    for name, a, (b, size) in zip(("Y", "dX", "dW_gate", "dW_up", "dW_down"), got, ref):
        _close(a, b, name, size, True)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
@pytest.mark.parametrize("T", [1, 40, 300])
def test_gated_activations(act, T, dtype):
    X, Wg, Wu, Wd = _gated_inputs(T, 136, 200, dtype, seed=20)
    dY = _rand(29, T, 136, dtype=dtype)
    Y, saved = dtp.gated_ffn(X, Wg, Wu, Wd, activation=act, save=True)
    got = (Y, *dtp.gated_ffn_backward(dY, X, Wg, Wu, Wd, saved, activation=act))
    ref = _gated_ref(X, Wg, Wu, Wd, None, act, dY)
    for name, a, (b, size) in zip(("Y", "dX", "dWg", "dWu", "dWd"), got, ref):
        _close(a, b, name, size, True)


def test_gradients_against_differences():
    """d<Y, dY>/dp along a random direction, by central differences of the fp64 formula and of the kernels' own
    fp32 forward pass.  A step of 1e-2 leaves the third derivative's (1e-2)^2 / 6, below 1e-3 of the slope at
    these scales, and the forward's rounding 1e-6 / 1e-2 of |Y|: 2e-2 of the gradient's scale is held."""
    T, d, N = 70, 48, 90
    P = list(_gated_inputs(T, d, N, F32, seed=40))
    dY = _rand(50, T, d, dtype=F32)
    _, saved = dtp.gated_ffn(*P, save=True)
    grads = dtp.gated_ffn_backward(dY, *P, saved)
    for k in range(4):
        v = _rand(60 + k, *P[k].shape, dtype=F32, std=1e-2)
        up, down = list(P), list(P)
        up[k], down[k] = P[k] + v, P[k] - v
        diff = ((dtp.gated_ffn(*up).double() - dtp.gated_ffn(*down).double()) * dY.double()).sum().item() / 2
        want = (grads[k].double() * v.double()).sum().item()
        scale = grads[k].double().norm().item() * v.double().norm().item() / math.sqrt(v.numel())
        assert abs(diff - want) <= 2e-2 * scale, (k, diff, want, scale)


def test_linear_gradient_against_differences():
    T, K, N = 60, 33, 50
    X, W, b = _rand(1, T, K, dtype=F32), _rand(2, N, K, dtype=F32, std=0.2), _rand(3, N, dtype=F32)
    dY = _rand(4, T, N, dtype=F32)
    for act in ("silu", "gelu"):
        _, Z = dtp.linear(X, W, b, activation=act, save=True)
        grads = dtp.linear_backward(dY, X, W, Z, activation=act, bias=True)
        P = [X, W, b]
        for k in range(3):
            v = _rand(70 + k, *P[k].shape, dtype=F32, std=1e-2)
            up, down = list(P), list(P)
            up[k], down[k] = P[k] + v, P[k] - v
            f = lambda q: dtp.linear(*q, activation=act).double()   # noqa: E731
            diff = ((f(up) - f(down)) * dY.double()).sum().item() / 2
            want = (grads[k].double() * v.double()).sum().item()
            scale = grads[k].double().norm().item() * v.double().norm().item() / math.sqrt(v.numel())
            assert abs(diff - want) <= 2e-2 * scale, (act, k)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_no_tokens(dtype):
    X, Wg, Wu, Wd = _gated_inputs(0, 64, 96, dtype)
    Y, saved = dtp.gated_ffn(X, Wg, Wu, Wd, save=True)
    assert Y.shape == (0, 64)
    grads = dtp.gated_ffn_backward(Y, X, Wg, Wu, Wd, saved)
    assert grads[0].shape == (0, 64) and all((g == 0).all() for g in grads[1:])
    Y, Z = dtp.linear(X, Wg, activation="gelu", save=True)
    dX, dW, db = dtp.linear_backward(Y, X, Wg, Z, activation="gelu", bias=True)
    assert Y.shape == (0, 96) and dX.shape == (0, 64) and (dW == 0).all() and (db == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 4, 40, 200, 600])
def test_repeatable_and_in_place_residual(T, dtype):
    """The same bits on every call, and with the residual overwritten by Y; nothing outside Y is written."""
    X, Wg, Wu, Wd = _gated_inputs(T, 264, 520, dtype, seed=3)
    R = _rand(5, T, 264, dtype=dtype)
    Y = dtp.gated_ffn(X, Wg, Wu, Wd, R)
    buf = torch.full(((T + 2) * 264,), 7.0, device=DEV, dtype=dtype)
    inner = buf[264:-264].view(T, 264)
    inner.copy_(R)
    dtp.gated_ffn(X, Wg, Wu, Wd, inner, Y=inner)
    assert torch.equal(inner, Y) and (buf[:264] == 7).all() and (buf[-264:] == 7).all()
    dY = _rand(6, T, 264, dtype=dtype)
    _, saved = dtp.gated_ffn(X, Wg, Wu, Wd, R, save=True)
    a = dtp.gated_ffn_backward(dY, X, Wg, Wu, Wd, saved)
    b = dtp.gated_ffn_backward(dY, X, Wg, Wu, Wd, saved)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("T", [1, 6, 50, 300])
def test_a_bad_token_stays_in_its_row(T):
    """NaN and infinity in one token reach that token's outputs alone."""
    X, Wg, Wu, Wd = _gated_inputs(T, 128, 256, BF16, seed=9)
    clean = dtp.gated_ffn(X, Wg, Wu, Wd)
    X2 = X.clone()
    X2[T // 2, 3] = float("nan")
    Y = dtp.gated_ffn(X2, Wg, Wu, Wd)
    keep = torch.arange(T, device=DEV) != T // 2
    assert torch.equal(Y[keep], clean[keep]) and torch.isnan(Y[T // 2]).all()
    X2[T // 2, 3] = float("inf")
    Y = dtp.gated_ffn(X2, Wg, Wu, Wd)
    assert torch.equal(Y[keep], clean[keep]) and not torch.isfinite(Y[T // 2]).any()


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_large_preactivations(act):
    """Saturated activations give the limits z and 0 and slopes 1 and 0, no NaN."""
    X = torch.tensor([[300.0], [-300.0], [3e4], [-3e4]], device=DEV, dtype=BF16)
    W = torch.ones((8, 1), device=DEV, dtype=BF16)
    Y, Z = dtp.linear(X, W, activation=act, save=True)
    assert torch.equal(Y.float(), X.float().clamp(min=0).expand(4, 8))
    dX, _, _ = dtp.linear_backward(torch.ones_like(Y), X, W, Z, activation=act)
    assert torch.equal(dX.flatten().cpu().float(), torch.tensor([8.0, 0.0, 8.0, 0.0]))


def test_other_stream_and_status():
    X, Wg, Wu, Wd = _gated_inputs(333, 256, 384, BF16, seed=11)
    ref = dtp.gated_ffn(X, Wg, Wu, Wd)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    ws = dtp.gated_ffn_workspace(333, 256, 384, BF16, DEV)
    s.wait_stream(torch.cuda.current_stream())
    Y = dtp.gated_ffn(X, Wg, Wu, Wd, workspace=ws, stream=s)
    s.synchronize()
    assert torch.equal(Y, ref)
    dtp.workspace_status(ws)


def test_graph_capture():
    """A captured call replays on new values in the same buffers."""
    X, Wg, Wu, Wd = _gated_inputs(40, 256, 384, BF16, seed=12)
    ws = dtp.gated_ffn_workspace(40, 256, 384, BF16, DEV)
    Y = dtp.gated_ffn(X, Wg, Wu, Wd, workspace=ws)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        dtp.gated_ffn(X, Wg, Wu, Wd, Y=Y, workspace=ws)
    X.copy_(_rand(99, 40, 256))
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(Y, dtp.gated_ffn(X, Wg, Wu, Wd))


def test_refusals():
    X, Wg, Wu, Wd = _gated_inputs(8, 64, 96, BF16)
    with pytest.raises(ValueError, match="activation"):
        dtp.gated_ffn(X, Wg, Wu, Wd, activation="tanh")
    with pytest.raises(TypeError):
        dtp.gated_ffn(X, Wg.float(), Wu, Wd)
    with pytest.raises(ValueError, match="W_down"):
        dtp.gated_ffn(X, Wg, Wu, Wd.t())
    with pytest.raises(ValueError, match="contiguous"):
        dtp.gated_ffn(X.t().contiguous().t(), Wg, Wu, Wd)
    with pytest.raises(ValueError, match="CUDA"):
        dtp.linear(X, Wg.cpu())
    with pytest.raises(TypeError):
        dtp.linear(X.half(), Wg.half())
    with pytest.raises(ValueError, match="Z"):
        dtp.linear_backward(torch.zeros(8, 96, device=DEV, dtype=BF16), X, Wg, activation="silu")
    with pytest.raises(dtp.DTPError) as e:
        dtp.gated_ffn(X, Wg, Wu, Wd, workspace=torch.empty(64, dtype=torch.uint8, device=DEV))
    assert e.value.status == dtp.DTP_ERR_WORKSPACE
    flat = torch.zeros(8 * 64 + 8, device=DEV, dtype=BF16)
    with pytest.raises(dtp.DTPError) as e:      # not on a 16-byte boundary
        dtp.gated_ffn(flat[1:1 + 8 * 64].view(8, 64), Wg, Wu, Wd)
    assert e.value.status == dtp.DTP_ERR_ARG


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_gradients_that_are_not_wanted(dtype):
    """Each gradient may be left out (NULL at the C ABI); the others keep their bits."""
    T, d, N = 150, 72, 136
    X, Wg, Wu, Wd = _gated_inputs(T, d, N, dtype, seed=30)
    dY = _rand(31, T, d, dtype=dtype)
    _, saved = dtp.gated_ffn(X, Wg, Wu, Wd, save=True)
    full = dtp.gated_ffn_backward(dY, X, Wg, Wu, Wd, saved)
    code = dtp.DTP_BF16 if dtype is BF16 else dtp.DTP_F32
    ws = dtp.gated_ffn_workspace(T, d, N, dtype, DEV, backward=True)
    stream = torch.cuda.current_stream().cuda_stream
    for skip in range(4):
        out = [None if i == skip else torch.empty_like(g) for i, g in enumerate(full)]
        st = dtp.lib().dtp_gated_ffn_backward(*(t.data_ptr() for t in (dY, X, Wg, Wu, Wd, *saved)), T, d, N, 1, code,
                                              *(None if t is None else t.data_ptr() for t in out), ws.data_ptr(), ws.numel(),
                                              stream)
        assert st == dtp.DTP_OK
        assert all(t is None or torch.equal(t, g) for t, g in zip(out, full))
    assert dtp.workspace_status(ws) == dtp.DTP_OK
    R = _rand(32, T, N, dtype=dtype)
    dX, dW, db = dtp.linear_backward(R, X, Wg, bias=True)
    ws = dtp.linear_workspace(T, d, N, dtype, DEV, backward=True)
    for skip in range(3):
        out = [None if i == skip else torch.empty_like(g) for i, g in enumerate((dX, dW, db))]
        st = dtp.lib().dtp_linear_backward(R.data_ptr(), X.data_ptr(), Wg.data_ptr(), None, T, d, N, 0, code,
                                           *(None if t is None else t.data_ptr() for t in out), ws.data_ptr(), ws.numel(),
                                           stream)
        assert st == dtp.DTP_OK
        assert all(t is None or torch.equal(t, g) for t, g in zip(out, (dX, dW, db)))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 2, 5, 40, 200])
def test_status_word_is_cleared(T, dtype):
    """An old code in the workspace's status word does not outlive a call that went well."""
    X, Wg, Wu, Wd = _gated_inputs(T, 136, 264, dtype, seed=33)
    for backward in (False, True):
        ws = dtp.gated_ffn_workspace(T, 136, 264, dtype, DEV, backward=backward)
        _, saved = dtp.gated_ffn(X, Wg, Wu, Wd, save=True)
        ws[:4].view(torch.int32).fill_(dtp.DTP_ERR_NOT_CONVERGED)
        if backward:
            dtp.gated_ffn_backward(X, X, Wg, Wu, Wd, saved, workspace=ws)
        else:
            dtp.gated_ffn(X, Wg, Wu, Wd, workspace=ws)
        assert dtp.workspace_status(ws) == dtp.DTP_OK
    ws = dtp.linear_workspace(T, 136, 264, dtype, DEV)
    ws[:4].view(torch.int32).fill_(dtp.DTP_ERR_NOT_CONVERGED)
    dtp.linear(X, Wg, workspace=ws)
    assert dtp.workspace_status(ws) == dtp.DTP_OK


def test_calls_in_a_row_on_one_workspace():
    """Launches overlap their predecessors' ends: a chain of calls that read and write the same buffers keeps its order."""
    X, Wg, Wu, Wd = _gated_inputs(300, 256, 512, BF16, seed=34)
    small, _, _, _ = _gated_inputs(2, 256, 512, BF16, seed=35)
    ws = dtp.gated_ffn_workspace(300, 256, 512, BF16, DEV, backward=True)
    ref = X
    for _ in range(4):
        ref = dtp.gated_ffn(ref, Wg, Wu, Wd, ref)
        torch.cuda.synchronize()
    refs = dtp.gated_ffn(dtp.gated_ffn(small, Wg, Wu, Wd), Wg, Wu, Wd)
    a, b = X.clone(), torch.empty_like(X)
    for _ in range(30):
        a.copy_(X)
        for i in range(4):
            dtp.gated_ffn(a, Wg, Wu, Wd, a, Y=b, workspace=ws)
            a, b = b, a
        s = dtp.gated_ffn(dtp.gated_ffn(small, Wg, Wu, Wd, workspace=ws), Wg, Wu, Wd, workspace=ws)
        assert torch.equal(a, ref) and torch.equal(s, refs)
