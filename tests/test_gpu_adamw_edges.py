"""The AdamW step at the ends of fp32's range."""
import pytest
import torch

from paper_2609_13846_gb300 import dtp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HYPER = dict(lr=3e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)
ROUND = 2.0 ** -24


@pytest.mark.parametrize("norm,limit", [(2e-39, 1e-39), (1e-42, 7e-43), (2.5e-39, 1e-41), (1.2e-38, 1e-38), (2e-38, 3e-39), (5e-39, 0.0),
                                        (1e-30, 1e-60), (3e38, 1e-290), (3e38, 5e-324), (1e10, 1e-300), (3e38, 1e38)])
@pytest.mark.parametrize("bits", [32, 8])
def test_norms_and_limits_at_the_ends(norm, limit, bits):
    """A factor below 1 is one wherever its two numbers lie: gradients of 0 stay 0, the others count times it."""
    g = torch.Generator(device=DEV).manual_seed(1)
    params = [torch.randn(700, generator=g, device=DEV)]
    size = torch.tensor(norm, device=DEV)
    grads = [torch.randn(700, generator=g, device=DEV) / 26.0 * size]        # of about that norm
    grads[0][::3] = 0.0
    state = dtp.adamw_state(params, bits=bits)
    before = params[0].clone()
    dtp.adamw_step(params, grads, state, norm=size, max_norm=limit, **HYPER)
    factor = limit / float(size)
    assert factor < 1.0
    m = 0.1 * grads[0].double() * factor
    held = dtp.adamw_moments(state)[0][0]
    assert (held[::3] == 0).all()
    if bits == 32:
        # subnormal numbers are off by 2^-150 each: the gradient in two parts, its factor, the moment
        assert ((held.double() - m).abs() <= 8 * ROUND * m.abs() + 4 * 2.0 ** -149).all()
    else:
        assert torch.isfinite(held).all()
        if norm * factor < 1e18:        # squares beyond fp32's range are held as NaN
            assert torch.isfinite(dtp.adamw_moments(state)[1][0]).all()
    if norm * factor < 1e-20:           # far below eps: the decay alone, a rounding of the factor and one of the product
        want = before.double() * (1 - HYPER["lr"] * HYPER["weight_decay"])
        assert ((params[0].double() - want).abs() <= 2.1 * ROUND * want.abs() + 1e-9).all()
    assert torch.isfinite(params[0]).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_a_factor_among_the_subnormal_numbers(bits):
    """Gradients of 1e20 and a limit of 1e-20: moments of 1e-22 are held like others, and the weights only decay."""
    g = torch.Generator(device=DEV).manual_seed(2)
    params = [torch.randn(n, generator=g, device=DEV) for n in (3000, 300)]
    grads = [torch.randn(n, generator=g, device=DEV) * 1e20 for n in (3000, 300)]
    norm = dtp.clip_grad_norm(grads, float("inf"))
    factor = 1e-20 / float(norm)
    assert factor < 1.2e-38
    state = dtp.adamw_state(params, bits=bits)
    before = [p.clone() for p in params]
    dtp.adamw_step(params, grads, state, norm=norm, max_norm=1e-20, **HYPER)
    for p, b, gr, held in zip(params, before, grads, dtp.adamw_moments(state)[0]):
        want = b.double() * (1 - HYPER["lr"] * HYPER["weight_decay"])
        assert ((p.double() - want).abs() <= 2.1 * ROUND * want.abs() + 1e-9).all()
        m = 0.1 * gr.double() * factor
        if bits == 32:
            assert ((held.double() - m).abs() <= 8 * ROUND * m.abs() + 1e-44).all()
            continue
        unit = torch.nn.functional.pad(m.abs(), (0, -m.numel() % 256)).view(-1, 256).amax(1).repeat_interleave(256)[:m.numel()] / 448
        step = torch.maximum(m.abs() / 8, 2.0 ** -9 * unit)
        assert ((held.double() - m).abs() <= 1.001 * step).all() and (held != 0).any()
