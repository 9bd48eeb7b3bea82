"""The global gradient norm and clipping against fp64.

Tolerances, before the first run: a chunk's squares are summed in fp32 by 512 threads (32 terms each, then a tree),
so the sum's relative error is below 45 roundings of 2^-24 and the norm's below half of that, 1.4e-6; 2e-6 is
held.  A scaled value is one fp32 product with a coefficient that is off by no more than that, rounded once:
2^-8 of bf16 (one step) and 2.5e-6 of fp32 are held."""
import math

import pytest
import torch

from paper_2609_13846_gb300 import dtp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def _tensors(sizes, dtypes, seed=0, std=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return [(torch.randn(n, generator=g, device=DEV) * std).to(dt) for n, dt in zip(sizes, dtypes)]


def _norm(ts):
    return math.sqrt(sum((t.double() ** 2).sum().item() for t in ts))


def _check(ts, max_norm, n, got, src):
    assert abs(n.item() - _norm(src)) <= 2e-6 * _norm(src)
    want = _norm(src)
    c = max_norm / want if want > max_norm else 1.0
    for a, b in zip(got, src):
        if c == 1.0:
            assert torch.equal(a, b)
        else:
            tol = 2.0 ** -8 if a.dtype is BF16 else 2.5e-6
            ref = b.double() * c
            assert ((a.double() - ref).abs() <= tol * ref.abs() + 1e-40).all()


@pytest.mark.parametrize("sizes", [[1], [0, 5, 0], [16384], [16385, 16383], [7, 100000, 3, 70001], [64] * 700,
                                   [3] * 1500 + [50000]])
@pytest.mark.parametrize("kind", ["bf16", "f32", "mixed"])
@pytest.mark.parametrize("ratio", [0.5, 3.0])
@pytest.mark.parametrize("inplace", [False, True])
def test_clip(sizes, kind, ratio, inplace):
    dts = {"bf16": [BF16], "f32": [F32], "mixed": [BF16, F32, F32]}[kind]
    ts = _tensors(sizes, [dts[i % len(dts)] for i in range(len(sizes))])
    src = [t.clone() for t in ts]
    max_norm = _norm(src) / ratio
    out = None if inplace else [torch.full_like(t, 9) for t in ts]
    n = dtp.clip_grad_norm(ts, max_norm, out=out)
    _check(ts, max_norm, n, ts if inplace else out, src)
    if not inplace:
        assert all(torch.equal(a, b) for a, b in zip(ts, src))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shift_in,shift_out", [(0, 0), (1, 1), (3, 3), (1, 2), (0, 5)])
def test_unaligned_views(dtype, shift_in, shift_out):
    """Packed views at any element offset; their neighbours are not touched."""
    n = 40001
    a = _tensors([n + 16], [dtype])[0]
    b = torch.full((n + 16,), 9.0, device=DEV, dtype=dtype)
    src, dst = a[shift_in:shift_in + n], b[shift_out:shift_out + n]
    limit = _norm([src]) / 2.7
    nrm = dtp.clip_grad_norm([src], limit, out=[dst])
    _check([src], limit, nrm, [dst], [src])
    assert (b[:shift_out] == 9).all() and (b[shift_out + n:] == 9).all()
    keep = a.clone()
    dtp.clip_grad_norm([src], limit)
    assert torch.equal(a[:shift_in], keep[:shift_in]) and torch.equal(a[shift_in + n:], keep[shift_in + n:])


@pytest.mark.parametrize("scale", [1e-30, 1e-24, 1e-12, 1.0, 1e15, 1e25, 1e30])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_squares_beyond_fp32(scale, dtype):
    """Norms whose squares overflow or vanish in fp32."""
    ts = _tensors([30000, 17], [dtype, dtype], std=scale)
    n = dtp.clip_grad_norm(ts, math.inf)
    assert abs(n.item() - _norm(ts)) <= 2e-6 * _norm(ts)


def test_zeros_and_limits():
    z = [torch.zeros(20000, device=DEV), torch.zeros(3, device=DEV, dtype=BF16)]
    assert dtp.clip_grad_norm(z, 0.0).item() == 0.0 and all((t == 0).all() for t in z)
    t = _tensors([1000], [F32])
    keep = t[0].clone()
    n = dtp.clip_grad_norm(t, math.inf)
    assert torch.equal(t[0], keep) and n.item() > 0
    dtp.clip_grad_norm(t, 0.0)
    assert (t[0] == 0).all()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_non_finite_norm_leaves_gradients(bad):
    ts = _tensors([50000, 300], [BF16, F32])
    ts[0][123] = bad
    src = [t.clone() for t in ts]
    out = [torch.zeros_like(t) for t in ts]
    n = dtp.clip_grad_norm(ts, 1.0, out=out)
    assert not math.isfinite(n.item()) and math.isnan(n.item()) == math.isnan(bad)
    for a, b, o in zip(ts, src, out):
        v = torch.int16 if a.dtype is BF16 else torch.int32
        assert torch.equal(a.view(v), b.view(v)) and torch.equal(o.view(v), b.view(v))
    dtp.clip_grad_norm(ts, 1.0)
    assert all(torch.equal(a[200:], b[200:]) for a, b in zip(ts, src))


def test_repeatable():
    ts = _tensors([100001, 5, 777777], [BF16, F32, F32])
    a = [dtp.clip_grad_norm(ts, math.inf).item() for _ in range(3)]
    assert a[0] == a[1] == a[2]


def test_large_tensor_offsets():
    """Offsets beyond 2^31 elements: the last chunk is read and scaled."""
    n = (1 << 31) + 20000
    t = torch.zeros(n, device=DEV, dtype=BF16)
    t[-1] = 3.0
    t[0] = 4.0
    norm = dtp.clip_grad_norm([t], 2.5)
    assert norm.item() == 5.0 and t[-1].item() == 1.5 and t[0].item() == 2.0


def test_refusals():
    t = _tensors([100], [F32])
    with pytest.raises(ValueError):
        dtp.clip_grad_norm([], 1.0)
    with pytest.raises(ValueError, match="CUDA"):
        dtp.clip_grad_norm([t[0].cpu()], 1.0)
    with pytest.raises(ValueError, match="contiguous"):
        dtp.clip_grad_norm([t[0][::2]], 1.0)
    with pytest.raises(TypeError):
        dtp.clip_grad_norm([t[0].half()], 1.0)
    with pytest.raises(ValueError, match="out"):
        dtp.clip_grad_norm(t, 1.0, out=[t[0].to(BF16)])
    for bad in (-1.0, math.nan):
        with pytest.raises(dtp.DTPError) as e:
            dtp.clip_grad_norm(t, bad)
        assert e.value.status == dtp.DTP_ERR_ARG
    with pytest.raises(dtp.DTPError) as e:
        dtp.clip_grad_norm(t, 1.0, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    assert e.value.status == dtp.DTP_ERR_WORKSPACE
