"""The loss where one token is far ahead: the logit that leads is taken out exactly, whatever its size."""
import math

import pytest
import torch

from paper_2609_13846_gb300 import dtp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
SHAPES = [(1, BF16), (40, BF16), (300, BF16), (5, F32), (20, F32), (70, F32)]


def _inputs(T, dtype, V, size, leaders, d=64):
    """Logits that are products of two numbers, so that they are exact: `size` at `leaders`, the others half of it at most."""
    g = torch.Generator(device=DEV).manual_seed(T)
    x = torch.zeros((T, d), device=DEV)
    w = torch.zeros((V, d), device=DEV)
    x[:, 3] = 2.0 ** torch.randint(0, 2, (T,), generator=g, device=DEV)
    w[:, 3] = (torch.rand(V, generator=g, device=DEV) - 1.0) * size
    w[torch.tensor(leaders, device=DEV), 3] = size
    return x.to(dtype), w.to(dtype)


@pytest.mark.parametrize("T,dtype", SHAPES)
@pytest.mark.parametrize("size", [60.0, 200.0, 1000.0, 15.0 * 2 ** 20, 1.0e30])
@pytest.mark.parametrize("V,leader", [(700, 100), (5003, 5002)])
def test_a_leader_has_no_loss_and_no_gradient(T, dtype, size, V, leader):
    """Where every other term is below 2^-24 / V of the leader's, lse is the leading logit to the bit, the leader's loss 0 and its
    gradient 0; at 60 the others add at most e^-60 V."""
    x, w = _inputs(T, dtype, V, size, [leader])
    w[:, 3] = torch.where(torch.arange(V, device=DEV) == leader, w[:, 3], -w[:, 3].abs())
    y = torch.full((T,), leader, device=DEV)
    z = x[:, 3].float() * w[leader, 3].float()
    loss, lse = dtp.linear_cross_entropy(x, w, y)
    assert torch.equal(lse, z)
    assert ((loss >= 0) & (loss <= 1e-20)).all()
    dx, dw = dtp.linear_cross_entropy_backward(torch.ones(T, device=DEV), x, w, y, lse)
    tiny = T * V * 1e-20 if size < 1e3 else 0.0
    assert (dw.float().abs() <= tiny).all() and (dx.float().abs() <= tiny * size).all()
    other = torch.full((T,), (leader + 1) % V, device=DEV)
    loss, _ = dtp.linear_cross_entropy(x, w, other)
    want = z.double() - x[:, 3].double() * w[(leader + 1) % V, 3].double()
    assert ((loss.double() - want).abs() <= 2.0 ** -24 * want).all()


@pytest.mark.parametrize("T,dtype", SHAPES)
@pytest.mark.parametrize("size", [200.0, 1000.0, 1.0e30])
def test_two_leaders_share_the_loss(T, dtype, size):
    """ln 2 each: a product with it, rounded, of 1 (twice an exponential of 0); where lse itself has room for it, so is p - 1 = -1/2."""
    x, w = _inputs(T, dtype, 900, size, [5, 831])
    w[:, 3] = torch.where(w[:, 3] == w[5, 3], w[:, 3], -w[:, 3].abs())
    for leader in (5, 831):
        loss, lse = dtp.linear_cross_entropy(x, w, torch.full((T,), leader, device=DEV))
        assert ((loss.double() - math.log(2.0)).abs() <= 2.0 ** -22).all()
        want = x[:, 3].double() * w[5, 3].double() + math.log(2.0)
        assert ((lse.double() - want).abs() <= 2.0 ** -23 * want).all()


@pytest.mark.parametrize("T,dtype", SHAPES)
@pytest.mark.parametrize("scale", [2.0, 50.0, 1000.0])
def test_no_loss_is_negative(T, dtype, scale):
    """A token's logit is at most the largest, and the sum of exponentials beside it at least one."""
    g = torch.Generator(device=DEV).manual_seed(T)
    x = torch.randn((T, 96), generator=g, device=DEV).to(dtype)
    w = (torch.randn((3001, 96), generator=g, device=DEV) * scale / 96 ** 0.5).to(dtype)
    best = (x.double() @ w.double().t()).argmax(1)
    loss, lse = dtp.linear_cross_entropy(x, w, best)
    assert (loss >= 0).all() and torch.isfinite(lse).all()
