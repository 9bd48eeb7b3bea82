"""The AdamW step's 8-bit states, bit for bit."""
import pytest
import torch

from paper_2609_13846_gb300 import dtp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
HYPER = dict(lr=3e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)


def _random(at, n, step):
    """The two numbers in [0, 1) by which the moments of elements at .. at + n - 1 are rounded, in 23 bits."""
    mask = 0xFFFFFFFF
    i = torch.arange(at, at + n, device=DEV)
    x = ((i & mask) + (i >> 32) * 0x85EBCA6B + step * 0x9E3779B9) & mask
    x = ((x ^ (x >> 16)) * 0x7FEB352D) & mask
    x = ((x ^ (x >> 15)) * 0x846CA68B) & mask
    x = x ^ (x >> 16)
    return [(h >> 9).float() * 2.0 ** -23 for h in (x, (x * 0x9E3779B1) & mask)]


def _blocks(x):
    return torch.nn.functional.pad(x, (0, -x.numel() % 256)).view(-1, 256)


def _hold(x, u, root):
    """(codes, scales) of x: whole steps of e4m3 above the largest / 448, rounded up where the fraction and u reach 1."""
    b = _blocks(x)
    top = b.abs().amax(1)
    some = top >= 2.0 ** -100
    up = torch.where(some, (1.0 / top) * 448.0, torch.zeros_like(top))
    a = (b.abs() * up[:, None]).view(-1)[:x.numel()]
    exponent = torch.floor(torch.log2(a.double().clamp(min=2.0 ** -6))).int()
    # log2 may land on the wrong side of a power of two
    exponent += (a.double() >= torch.ldexp(torch.ones_like(a, dtype=torch.float64), exponent + 1)).int()
    exponent -= (a.double() < torch.ldexp(torch.ones_like(a, dtype=torch.float64), exponent)).int() * (exponent > -6).int()
    steps = torch.ldexp(a, 3 - exponent)                      # exact: 8 to 16 in normal codes, below 8 in subnormal ones
    code = (torch.floor(steps + u).int() + (exponent + 6) * 8).clamp(max=0x7E)
    if root:
        code = torch.where((code == 0) & (x > 0), torch.ones_like(code), code)
    code = code + 128 * torch.signbit(x).int()
    return code.to(torch.uint8), torch.where(some, top * torch.tensor(1.0 / 448.0, device=DEV), torch.zeros_like(top))


def _emulated(code, scale, grad, at, step, betas):
    """The 8-bit states after a step, each operation rounded to fp32 by itself: (m, m_scale, v, v_scale)."""
    def held(k):
        return (_blocks(code[k].view(torch.float8_e4m3fn).float()) * scale[k][:, None]).view(-1)[:grad.numel()]

    g = grad.float()
    m = held("m") * betas[0] + g * (1.0 - betas[0])
    old = held("v")
    v = old * old * betas[1] + g * g * (1.0 - betas[1])
    u, w = _random(at, grad.numel(), step)
    return *_hold(m, u, False), *_hold(v.sqrt(), w, True)


@pytest.mark.parametrize("sizes", [[1, 255, 256, 257, 70_001], [300_000]], ids=["odd", "large"])
@pytest.mark.parametrize("param,grad", [(F32, BF16), (BF16, F32)])
def test_codes_are_those_of_the_formula(sizes, param, grad):
    """The states' arithmetic is fixed to the bit: separately rounded fp32 operations anywhere give the same codes and scales.
    Gradients of all sizes within a block, so that a tenth of the codes are subnormal ones."""
    g = torch.Generator(device=DEV).manual_seed(3)
    params = [torch.randn(n, generator=g, device=DEV).to(param) for n in sizes]
    state = dtp.adamw_state(params, bits=8)
    for t in range(1, 5):
        grads = [(torch.randn(n, generator=g, device=DEV) * torch.exp(2.0 * torch.randn(n, generator=g, device=DEV)) * 1e-3).to(grad)
                 for n in sizes]
        before = [({k: state[k][i].view(torch.uint8).clone() for k in ("m", "v")}, {k: state[k + "_scale"][i].clone() for k in ("m", "v")})
                  for i in range(len(sizes))]
        dtp.adamw_step(params, grads, state, lr=1e-3, betas=(0.9, 0.95))
        for i, (code, scale) in enumerate(before):
            want = _emulated(code, scale, grads[i], 0, t, (0.9, 0.95))
            got = (state["m"][i].view(torch.uint8), state["m_scale"][i], state["v"][i].view(torch.uint8), state["v_scale"][i])
            for k, a, b in zip(("m", "m_scale", "v", "v_scale"), got, want):
                assert torch.equal(a, b), (t, i, k, int((a != b).sum()))
    assert ((state["m"][-1].view(torch.uint8) & 0x78) == 0).any()


def test_codes_beyond_32_bits():
    """The hash takes the element's whole index: the codes at both ends of a tensor of more than 2^32 elements."""
    n = (1 << 32) + 300
    p, g = (torch.zeros(n, dtype=BF16, device=DEV) for _ in range(2))
    gen = torch.Generator(device=DEV).manual_seed(4)
    first = n // 256 * 256 - 512
    ends = ((0, 1024), (first, n))
    for a, b in ends:
        g[a:b] = torch.randn(b - a, generator=gen, device=DEV).to(BF16)
    state = dtp.adamw_state([p], bits=8)
    dtp.adamw_step([p], [g], state, **HYPER)
    for a, b in ends:
        k = -(-(b - a) // 256)
        zero = {x: torch.zeros(b - a, dtype=torch.uint8, device=DEV) for x in ("m", "v")}, {x: torch.zeros(k, device=DEV) for x in ("m", "v")}
        want = _emulated(*zero, g[a:b], a, 1, HYPER["betas"])
        got = (state["m"][0][a:b].view(torch.uint8), state["m_scale"][0][a // 256:a // 256 + k], state["v"][0][a:b].view(torch.uint8),
               state["v_scale"][0][a // 256:a // 256 + k])
        assert all(torch.equal(x, y) for x, y in zip(got, want)), a
