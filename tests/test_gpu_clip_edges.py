"""The gradient norm with infinities, norms beyond fp32, and coefficients below fp32's normal numbers."""
import math

import pytest
import torch

from paper_2609_13846_gb300 import dtp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
TYPES = pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
BAD = pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])


def _expect(norm, bad):
    assert math.isnan(norm.item()) if math.isnan(bad) else norm.item() == math.inf


@TYPES
@BAD
@pytest.mark.parametrize("n", [100, 5000, 300_001, 100_000_003])
def test_bad_element_anywhere(n, bad, dtype):
    """An infinity makes the norm +inf and a NaN makes it NaN, wherever it lies: before the first 16-byte word (the views
    start one element past one), in the first words, in the middle, after the last word.  The gradients stay."""
    g = torch.full((n + 1,), 0.5, device=DEV, dtype=dtype)[1:]
    for at in (0, 9, n // 2, n - 10, n - 1):
        g[at] = bad
        _expect(dtp.clip_grad_norm([g], 1.0), bad)
        g[at] = 0.5
        assert (g == 0.5).all()


@BAD
@pytest.mark.parametrize("at", [0, 1, 750, 1499])
def test_bad_element_among_many_tensors(at, bad):
    ts = [torch.full((3,), 0.5, device=DEV, dtype=F32 if i % 3 else BF16) for i in range(1500)]
    ts[at][1] = bad
    _expect(dtp.clip_grad_norm(ts, 1.0), bad)


def test_infinities_of_both_signs():
    g = torch.full((500_000,), 0.5, device=DEV)
    g[3], g[400_000] = math.inf, -math.inf
    _expect(dtp.clip_grad_norm([g], 1.0), math.inf)
    g[499_999] = math.nan
    _expect(dtp.clip_grad_norm([g], 1.0), math.nan)


@TYPES
@pytest.mark.parametrize("inplace", [True, False])
def test_finite_gradients_whose_norm_is_not(dtype, inplace):
    """sqrt(1000) 3e38 is no fp32 number: the norm reads infinite, and what the caller will skip is not scaled."""
    ts = [torch.full((n,), 3e38, device=DEV, dtype=dtype) for n in (990, 10)]
    keep = [t.clone() for t in ts]
    out = None if inplace else [torch.zeros_like(t) for t in ts]
    assert dtp.clip_grad_norm(ts, 1.0, out=out).item() == math.inf
    assert all(torch.equal(a, b) for a, b in zip(ts, keep))
    assert inplace or all(torch.equal(a, b) for a, b in zip(out, keep))


@TYPES
@pytest.mark.parametrize("max_norm", [1.0, 1e-6, 1e-20, 1e-35])
@pytest.mark.parametrize("scale", [1.0, 1e20, 1e36])
def test_small_factors(max_norm, scale, dtype):
    """max_norm / n from 1e-3 to 1e-74: below fp32's normal numbers and below all of them.  The norm is held to 2e-6 as in the
    other tests; a scaled value is off by the norm's error and one rounding (2^-8, 2^-23), or half of the smallest
    subnormal number of its type."""
    g = torch.Generator(device=DEV).manual_seed(3)
    ts = [(torch.rand(n, generator=g, device=DEV) * scale).to(dtype) for n in (1000, 37)]
    src = [t.double() for t in ts]
    n = math.sqrt(sum((t ** 2).sum().item() for t in src))
    assert abs(dtp.clip_grad_norm(ts, max_norm).item() - n) <= 2e-6 * n
    u, least = (2.0 ** -8, 2.0 ** -133) if dtype is BF16 else (2.0 ** -23, 2.0 ** -149)
    for a, b in zip(ts, src):
        ref = b * (torch.tensor(max_norm, dtype=F32).item() / n)
        assert ((a.double() - ref).abs() <= (u + 2.1e-6) * ref + 0.51 * least).all()
