"""The distillation example: a permuted layer is the dense one, its gradients are autograd's, and it learns."""
import pytest
import torch

from paper_2609_13846_gb300 import distill, dtp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _layer(T=300):
    return distill.make_layer(256, 384, 8, 4, 32, T, seed=5, device=DEV)


def test_permuted_layer_computes_the_same_function():
    """Only the order of the sums changes: each output is rounded three times on the way (r, H, Y), so two runs differ by
    a few bf16 roundings of the largest value on the path."""
    dense, W, attn, x = _layer()
    y, rms = distill.layer_forward(dense, attn, x)
    A = torch.rand((4, 384), device=DEV)
    lay = dtp.search_layout(A, D=2, iters=5)
    perm, heads, _ = dtp.apply_layout(W, lay["h"][None], lay["nu"][None], D=2, head_dim=32)
    group = attn.view(300, 4, -1)[:, heads[0].long()].reshape(300, -1).contiguous()
    w = dict(o=perm["o"][0], gate=perm["gate"][0], up=perm["up"][0], down=perm["down"][0], gamma=dense["gamma"])
    y2, rms2 = distill.layer_forward(w, group, x)
    assert (y.float() - y2.float()).abs().max() <= 4 * 2.0 ** -8 * y.float().abs().max()
    assert (rms - rms2).abs().max() <= 2.0 ** -8 * rms.max()


def test_gradients_are_autograds():
    """Against torch's autograd in fp64 on the same bf16 weights.  The path rounds r, h, H, dG, dU, dr and each gradient
    once (2^-8 sqrt(1/5) of a value on average): 7 roundings in quadrature are below 1% of a gradient's norm."""
    dense, _, attn, x = _layer()
    y, _, kept = distill.layer_forward(dense, attn, x, save=True)
    dy = torch.randn(y.shape, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).to(torch.bfloat16)
    got = distill.layer_backward(dense, dy, kept)
    p = {k: v.double().requires_grad_() for k, v in dict(dense, attn=attn, x=x).items()}
    r = p["x"] + p["attn"] @ p["o"].t()
    h = r * torch.rsqrt(r.square().mean(-1, keepdim=True) + distill.EPS) * p["gamma"]
    out = r + (torch.nn.functional.silu(h @ p["gate"].t()) * (h @ p["up"].t())) @ p["down"].t()
    ref = torch.autograd.grad(out, list(p.values()), dy.double())
    for (k, _), g in zip(p.items(), ref):
        assert (got[k].double() - g).norm() <= 1e-2 * g.norm(), k


def test_a_perturbed_layer_learns():
    """Gradient descent with the rate lr and the clipped gradient c g lowers the loss by lr c |g|^2 (1 - e) a step, where e, the
    curvature's share lr c g^T H g / 2 |g|^2, is below 1 as long as the rate is below 2 / the largest curvature; with the rate
    here the loss falls in every step, and over all of them by between a half of the first-order sum and all of it (a
    tenth more for the rounding of the weights that the layer runs on)."""
    dense, _, attn, x = _layer()
    teacher, _ = distill.layer_forward(dense, attn, x)
    gen = torch.Generator(device=DEV).manual_seed(2)
    master = {k: v.float() + 0.3 * float(v.float().std()) * torch.randn(v.shape, generator=gen, device=DEV)
              for k, v in dense.items()}
    lr, limit = 5e-3, 10.0
    losses, first_order = [], 0.0
    for _ in range(26):
        loss, norm = distill.distill_step(master, teacher, attn, x, lr=lr, max_norm=limit)
        losses.append(float(loss))
        first_order += lr * float(norm) * min(float(norm), limit)
    first_order -= lr * float(norm) * min(float(norm), limit)       # the last step's loss is not seen
    assert all(b < a for a, b in zip(losses, losses[1:]))
    assert 0.5 * first_order <= losses[0] - losses[-1] <= 1.1 * first_order


def test_a_bad_step_changes_nothing():
    dense, _, attn, x = _layer(40)
    teacher, _ = distill.layer_forward(dense, attn, x)
    master = {k: v.float().clone() for k, v in dense.items()}
    keep = {k: v.clone() for k, v in master.items()}
    attn[3, 5] = float("inf")
    _, norm = distill.distill_step(master, teacher, attn, x, lr=1e-2, max_norm=1.0)
    assert not torch.isfinite(norm) and all(torch.equal(master[k], keep[k]) for k in keep)
