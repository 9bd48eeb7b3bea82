"""The RMS norm and its gradients against the formulas in fp64."""
import pytest
import torch

from paper_2609_13846_gb300 import dtp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-6
ROUND = 2.0 ** -24       # half a step of fp32


def _inputs(T, d, dtype, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x, dy, dres = (torch.randn((T, d), generator=g, device=DEV) for _ in range(3))
    x[:, : max(1, d // 64)] *= 20.0
    gamma = 1.0 + 0.3 * torch.randn(d, generator=g, device=DEV)
    return x.to(dtype), gamma, dy.to(dtype), dres.to(dtype)


def _half(dtype):
    return torch.finfo(dtype).eps / 2


def _sum_error(d):
    """Relative error of a sum of d terms of one sign by 32 lanes or more, and of what follows it."""
    return (d / 32 + 24) * ROUND


def _check(x, gamma, dy, dres, y, rms, dx, dgamma):
    X, G, D = x.double(), gamma.double(), dy.double()
    R = (X.square().mean(-1) + EPS).sqrt()
    n = X / R[:, None]
    half, e = _half(x.dtype), _sum_error(x.shape[1])
    assert ((rms.double() - R).abs() <= e * R).all()
    assert ((y.double() - n * G).abs() <= (half + e) * 1.01 * (n * G).abs() + 1e-38).all()
    if dx is None:
        return
    dn = D * G
    mean = (dn * n).mean(-1, keepdim=True)
    want = (dn - n * mean) / R[:, None]
    size = (dn.abs() + n.abs() * (dn * n).abs().mean(-1, keepdim=True)) / R[:, None]
    if dres is not None:
        want, size = want + dres.double(), size + dres.double().abs()
    assert ((dx.double() - want).abs() <= half * want.abs() + 4 * e * size).all()
    # runs of at most 256 tokens in fp32, added in fp64
    T = x.shape[0]
    assert ((dgamma.double() - (D * n).sum(0)).abs() <= (min(T, 256) + 16 + x.shape[1] / 32) * ROUND * (D * n).abs().sum(0)).all()


@pytest.mark.parametrize("T,d", [(1, 1), (1, 7), (1, 4096), (2, 8), (3, 1001), (5, 1024), (33, 1536), (700, 64), (1003, 1537),
                                 (64, 4104), (9, 8192), (4, 8200), (3, 20001), (1, 1 << 20), (2049, 256), (40000, 24)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_formula(T, d, dtype):
    x, gamma, dy, dres = _inputs(T, d, dtype)
    y, rms = dtp.rms_norm(x, gamma, eps=EPS)
    for r in (None, dres):
        dx, dgamma = dtp.rms_norm_backward(dy, x, gamma, rms, dresidual=r)
        _check(x, gamma, dy, r, y, rms, dx, dgamma)


@pytest.mark.parametrize("T,d", [(37, 264), (300, 2048)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shift", [0, 1, 4])
def test_views_into_larger_tensors(T, d, dtype, shift):
    """Rows that start on any element: the same values bit for bit as aligned ones give, and nothing around them is written."""
    x, gamma, dy, dres = _inputs(T, d, dtype)

    def view(t):
        big = torch.full((t.numel() + 16,), 7.0, dtype=t.dtype, device=DEV)
        v = big[shift:shift + t.numel()].view(t.shape)
        v.copy_(t)
        return big, v

    y, rms = dtp.rms_norm(x, gamma)
    dx, dgamma = dtp.rms_norm_backward(dy, x, gamma, rms, dresidual=dres)
    big, out = view(torch.zeros_like(x))
    y2, rms2 = dtp.rms_norm(view(x)[1], view(gamma)[1], Y=out)
    assert y2 is out and torch.equal(y, y2) and torch.equal(rms, rms2)
    assert (big[:shift] == 7.0).all() and (big[shift + x.numel():] == 7.0).all()
    dx2, dgamma2 = dtp.rms_norm_backward(view(dy)[1], view(x)[1], view(gamma)[1], view(rms)[1], dresidual=view(dres)[1])
    assert torch.equal(dx, dx2) and torch.equal(dgamma, dgamma2)


def test_in_place_and_no_tokens():
    x, gamma, dy, _ = _inputs(50, 136, torch.bfloat16)
    y, rms = dtp.rms_norm(x, gamma)
    z = x.clone()
    assert torch.equal(dtp.rms_norm(z, gamma, Y=z)[0], y) and torch.equal(z, y)
    none = torch.empty((0, 136), dtype=torch.bfloat16, device=DEV)
    y, rms = dtp.rms_norm(none, gamma)
    assert y.shape == (0, 136) and rms.shape == (0,)
    dx, dgamma = dtp.rms_norm_backward(none, none, gamma, rms)
    assert dx.shape == (0, 136) and (dgamma == 0).all()


@pytest.mark.parametrize("d", [64, 3000, 9000])
def test_extreme_rows(d):
    """Squares beyond fp32's range, rows of zeros, infinities and NaNs stay in their own rows."""
    x, gamma, dy, _ = _inputs(6, d, torch.float32)
    x[1] *= 1e25
    x[2] *= 1e-30
    x[3] = 0.0
    x[4, 5] = float("inf")
    x[5, 0] = float("nan")
    y, rms = dtp.rms_norm(x, gamma, eps=EPS)
    some = slice(0, 4)
    _check(x[some], gamma, dy[some], None, y[some], rms[some], None, None)
    assert torch.isinf(rms[4]) and torch.isnan(y[4, 5]) and (y[4, :5] == 0).all()
    assert torch.isnan(rms[5]) and torch.isnan(y[5]).all()


def test_gradient_against_differences():
    """The directional derivative of <y, dy>: central differences in fp64 of the formula against the library's gradients; the
    second differences of these smooth rows are below 1e-6 of the first at this step."""
    x, gamma, dy, _ = _inputs(5, 96, torch.float32)
    _, rms = dtp.rms_norm(x, gamma, eps=EPS)
    dx, dgamma = dtp.rms_norm_backward(dy, x, gamma, rms)

    def value(x, gamma):
        return (x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * gamma * dy.double()).sum()

    g = torch.Generator(device=DEV).manual_seed(9)
    for wx, wg in ((1.0, 0.0), (0.0, 1.0)):
        ax = wx * torch.randn(x.shape, generator=g, device=DEV, dtype=torch.float64)
        ag = wg * torch.randn(gamma.shape, generator=g, device=DEV, dtype=torch.float64)
        h = 1e-4
        diff = (value(x.double() + h * ax, gamma.double() + h * ag) - value(x.double() - h * ax, gamma.double() - h * ag)) / (2 * h)
        got = (dx.double() * ax).sum() + (dgamma.double() * ag).sum()
        size = (dx.double() * ax).abs().sum() + (dgamma.double() * ag).abs().sum()
        assert abs(got - diff) <= 1e-5 * size


def test_streams_and_graphs():
    x, gamma, dy, dres = _inputs(257, 1000, torch.bfloat16)
    y, rms = dtp.rms_norm(x, gamma)
    dx, dgamma = dtp.rms_norm_backward(dy, x, gamma, rms, dresidual=dres)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y2, rms2 = dtp.rms_norm(x, gamma, stream=side)
    dx2, dgamma2 = dtp.rms_norm_backward(dy, x, gamma, rms2, dresidual=dres, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, y2) and torch.equal(dx, dx2) and torch.equal(dgamma, dgamma2)
    ws = dtp.rms_norm_workspace(257, 1000, torch.bfloat16, DEV)
    graph = torch.cuda.CUDAGraph()
    a, b = x.clone(), dy.clone()
    with torch.cuda.graph(graph):
        y3, rms3 = dtp.rms_norm(a, gamma)
        dx3, dgamma3 = dtp.rms_norm_backward(b, a, gamma, rms3, dresidual=dres, workspace=ws)
    a.copy_(x.flip(0))
    b.copy_(dy.flip(0))
    graph.replay()
    want, wrms = dtp.rms_norm(x.flip(0).contiguous(), gamma)
    wdx, wdgamma = dtp.rms_norm_backward(b, a, gamma, wrms, dresidual=dres)
    assert torch.equal(y3, want) and torch.equal(dx3, wdx) and torch.equal(dgamma3, wdgamma)


@pytest.mark.parametrize("d", [200, 1001, 4096, 9000])
@pytest.mark.parametrize("over", ["dY", "dresidual"])
def test_gradient_in_place_of_an_input(d, over):
    """At the C ABI dX may be dY or the residual's gradient; either output may be left out."""
    x, gamma, dy, dres = _inputs(70, d, torch.bfloat16)
    _, rms = dtp.rms_norm(x, gamma)
    want, wgamma = dtp.rms_norm_backward(dy, x, gamma, rms, dresidual=dres)
    ws = dtp.rms_norm_workspace(70, d, torch.bfloat16, DEV)

    def call(dy, dres, dx, dgamma):
        st = dtp.lib().dtp_rms_norm_backward(dy.data_ptr(), x.data_ptr(), gamma.data_ptr(), rms.data_ptr(), dres.data_ptr(), 70, d,
                                             dtp.DTP_BF16, None if dx is None else dx.data_ptr(),
                                             None if dgamma is None else dgamma.data_ptr(), ws.data_ptr(), ws.numel(),
                                             torch.cuda.current_stream().cuda_stream)
        assert st == dtp.DTP_OK

    a, b, dgamma = dy.clone(), dres.clone(), torch.zeros_like(gamma)
    dx = a if over == "dY" else b
    call(a, b, dx, dgamma)
    assert torch.equal(dx, want) and torch.equal(dgamma, wgamma)
    alone, galone = torch.zeros_like(x), torch.zeros_like(gamma)
    call(dy, dres, alone, None)
    call(dy, dres, None, galone)
    assert torch.equal(alone, want) and torch.equal(galone, wgamma)


def test_offsets_beyond_32_bits():
    """More than 2^31 elements: the last rows are those of a call on them alone, bit for bit."""
    T, d = 270_000, 8192
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.empty((T, d), dtype=torch.bfloat16, device=DEV)
    for t in range(0, T, 30_000):
        x[t:t + 30_000] = torch.randn((30_000, d), generator=g, device=DEV)
    assert x.numel() > 1 << 31
    gamma = 1.0 + 0.1 * torch.randn(d, generator=g, device=DEV)
    y, rms = dtp.rms_norm(x, gamma)
    last, lrms = dtp.rms_norm(x[-5:].contiguous(), gamma)
    assert torch.equal(y[-5:], last) and torch.equal(rms[-5:], lrms)
    dx, dgamma = dtp.rms_norm_backward(y, x, gamma, rms)
    ldx, _ = dtp.rms_norm_backward(last, x[-5:].contiguous(), gamma, lrms)
    assert torch.equal(dx[-5:], ldx)
    want = sum((y[t:t + 30_000].double() * x[t:t + 30_000].double() / rms[t:t + 30_000, None].double()).sum(0) for t in range(0, T, 30_000))
    assert ((dgamma.double() - want).abs() <= 600 * ROUND * want.abs()).all()       # terms of one sign
