"""The AdamW step against the formula in fp64, with states in 32 and in 8 bits."""
import math

import pytest
import torch

from paper_2609_13846_gb300 import dtp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
HYPER = dict(lr=3e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)
ROUND = 2.0 ** -24


def _tensors(sizes, param, grad, seed=0, shift=0, std=1e-2):
    """(params, grads): views that start ``shift`` elements into a packed buffer."""
    g = torch.Generator(device=DEV).manual_seed(seed)

    def pack(dtype, scale):
        flat = (torch.randn(sum(sizes) + shift, generator=g, device=DEV) * scale).to(dtype)
        out, at = [], shift
        for n in sizes:
            out.append(flat[at:at + n])
            at += n
        return out

    return pack(param, 0.05), pack(grad, std)


def _exact(p, g, m, v, t, lr, betas, eps, weight_decay, factor=1.0):
    """(p, m, v) after the step in fp64, and the size of p's update."""
    g = g.double() * factor
    m = betas[0] * m.double() + (1 - betas[0]) * g
    v = betas[1] * v.double() + (1 - betas[1]) * g * g
    u = lr * (m / (1 - betas[0] ** t)) / ((v / (1 - betas[1] ** t)).sqrt() + eps)
    return p.double() * (1 - lr * weight_decay) - u, m, v, u.abs() + p.double().abs()


def _check_params(p, want, size, before):
    """fp32: a dozen roundings of the update and of the weight, and the powers' in fp64.  bf16: a whole step, since they are rounded up or
    down, of the larger of the values before and after that rounding."""
    tol = 16 * ROUND * size
    if p.dtype == BF16:
        tol = tol + torch.finfo(BF16).eps * torch.maximum(want.abs(), p.double().abs())
    assert ((p.double() - want).abs() <= tol).all()


SIZES = [[1], [255, 0, 256, 257], [5, 1000, 3, 70001, 8], [4096] * 70, [100] * 900 + [131072]]


@pytest.mark.parametrize("sizes", SIZES, ids=[str(len(s)) for s in SIZES])
@pytest.mark.parametrize("param,grad", [(F32, F32), (F32, BF16), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("bits", [32, 8])
def test_formula_over_steps(sizes, param, grad, bits):
    params, grads = _tensors(sizes, param, grad)
    state = dtp.adamw_state(params, bits=bits)
    for t in range(1, 4):
        m, v = ([x.clone() for x in y] for y in dtp.adamw_moments(state))
        before = [p.clone() for p in params]
        held = [g.clone() for g in grads]
        dtp.adamw_step(params, grads, state, **HYPER)
        assert int(state["step"]) == t
        m2, v2 = dtp.adamw_moments(state)
        for i in range(0, len(sizes), max(1, len(sizes) // 8)):
            want, em, ev, size = _exact(before[i], grads[i], m[i], v[i], t, **HYPER)
            _check_params(params[i], want, size, before[i])
            assert torch.equal(grads[i], held[i])
            sm = (HYPER["betas"][0] * m[i].double()).abs() + (1 - HYPER["betas"][0]) * grads[i].double().abs()
            if bits == 32:
                assert ((m2[i].double() - em).abs() <= 4 * ROUND * sm).all()
                assert ((v2[i].double() - ev).abs() <= 5 * ROUND * ev + 1e-45).all()
            else:
                _check_held(m2[i], em, 0)
                _check_held(v2[i].double().sqrt(), ev.sqrt(), 1)
        for g in grads:
            g.mul_(-0.7)


def _check_held(got, want, floor):
    """Held within a step of e4m3 (an eighth of the value at most, 2^-9 of the scale's unit below) of the wanted value, give or
    take its own rounding; a positive root (``floor``) is at least one step."""
    n = want.numel()
    pad = torch.nn.functional.pad(want.abs(), (0, -n % 256)).view(-1, 256).amax(1)
    unit = (pad / 448).repeat_interleave(256)[:n]
    step = torch.maximum(2.0 ** (torch.floor(torch.log2(want.abs() / unit + 1e-300)) - 3), torch.full_like(unit, 2.0 ** -9)) * unit
    assert ((got.double() - want).abs() <= step * 1.001).all()
    if floor:
        assert (got[(want > 0) & (unit > 0)] > 0).all()


@pytest.mark.parametrize("shift", [1, 2, 3, 5, 8])
@pytest.mark.parametrize("bits", [32, 8])
def test_packed_views(shift, bits):
    """Tensors that start on any element give the same values as aligned ones, bit for bit, and their neighbours stay."""
    sizes = [1000, 7, 2049]
    outs = []
    for s in (0, shift):
        params, grads = _tensors(sizes, F32, BF16)
        if s:
            flat = torch.full((sum(sizes) + 3 * s + 9,), 3.0, device=DEV)
            at, moved = s, []
            for p in params:
                moved.append(flat[at:at + p.numel()])
                moved[-1].copy_(p)
                at += p.numel() + 1
            gflat = torch.zeros(sum(sizes) + s, device=DEV, dtype=BF16)
            gs, at = [], s
            for g in grads:
                gs.append(gflat[at:at + g.numel()])
                gs[-1].copy_(g)
                at += g.numel()
            params, grads = moved, gs
        copies = [torch.full((p.numel() + 9,), 5.0, device=DEV, dtype=BF16)[s:s + p.numel()] for p in params]
        state = dtp.adamw_state(params, bits=bits)
        for k in ("m", "v"):
            state[k] = [torch.zeros(n + 16, dtype=x.dtype if bits == 32 else torch.uint8, device=DEV)[s:s + n]
                        for x, n in zip(state[k], sizes)]
            if bits == 8:
                state[k] = [x.view(torch.float8_e4m3fn) for x in state[k]]
        for _ in range(2):
            dtp.adamw_step(params, grads, state, copies=copies, **HYPER)
        if s:
            assert flat[:s].eq(3.0).all() and flat[s + 1000] == 3.0 and flat[s + 1008] == 3.0
        m, v = dtp.adamw_moments(state)
        outs.append([x.clone() for x in params + copies + m + v])
        for p, c in zip(params, copies):
            assert torch.equal(c, p.to(BF16))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("ratio", [0.5, 4.0, 1e30])
def test_clipping_by_a_norm(bits, ratio):
    """Gradients of a norm above the limit count times limit / norm, also where that is among fp32's subnormal numbers."""
    std = 1e-2 if ratio < 1e20 else 1e20
    params, grads = _tensors([3000, 300], F32, F32, std=std)
    norm = dtp.clip_grad_norm(grads, math.inf)
    limit = float(norm) / ratio if ratio < 1e20 else 1e-20
    if ratio >= 1e20:
        assert limit / float(norm) < 1.2e-38
    factor = min(1.0, limit / float(norm))
    hyper = dict(HYPER, eps=1e-30)
    state = dtp.adamw_state(params, bits=bits)
    before = [p.clone() for p in params]
    dtp.adamw_step(params, grads, state, norm=norm, max_norm=limit, **hyper)
    for p, b, g, z in zip(params, before, grads, state["m"]):
        zero = torch.zeros_like(p)
        # g^2 of the smallest gradients is among fp32's subnormal numbers: off by 2^-150
        want, em, ev, size = _exact(b, g, zero, zero, 1, factor=factor, **hyper)
        some = ev > 1e-36 if ratio < 1e20 else torch.zeros_like(ev, dtype=torch.bool)
        _check_params(p[some], want[some], size[some], b[some])
        if bits == 32:
            assert ((z.double() - em).abs() <= 8 * ROUND * em.abs() + 2e-45).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_a_norm_that_is_not_finite_changes_nothing(bits, value):
    params, grads = _tensors([3000, 300], F32, BF16)
    state = dtp.adamw_state(params, bits=bits)
    copies = [torch.zeros_like(p, dtype=BF16) for p in params]
    dtp.adamw_step(params, grads, state, copies=copies, **HYPER)
    held = [x.clone() for x in params + copies + list(dtp.adamw_moments(state)[0]) + list(dtp.adamw_moments(state)[1])]
    grads[1][7] = value
    norm = dtp.clip_grad_norm(grads, math.inf)
    dtp.adamw_step(params, grads, state, copies=copies, norm=norm, max_norm=1.0, **HYPER)
    now = params + copies + list(dtp.adamw_moments(state)[0]) + list(dtp.adamw_moments(state)[1])
    assert all(torch.equal(a, b) for a, b in zip(held, now)) and int(state["step"]) == 1
    grads[1][7] = 0.0
    dtp.adamw_step(params, grads, state, copies=copies, norm=dtp.clip_grad_norm(grads, math.inf), max_norm=1.0, **HYPER)
    assert int(state["step"]) == 2 and not torch.equal(held[0], params[0])


@pytest.mark.parametrize("bits", [32, 8])
def test_values_that_are_not_finite_stay_where_they_are(bits):
    """Without a norm a bad gradient spoils its own parameter and no other of its block."""
    params, grads = _tensors([700], F32, F32)
    clean = [params[0].clone()], [grads[0].clone()]
    grads[0][10], grads[0][300], grads[0][301] = float("nan"), float("inf"), 1e30
    bad = torch.zeros(700, dtype=torch.bool, device=DEV)
    bad[[10, 300, 301]] = True
    clean[1][0][bad] = 0.0
    states = [dtp.adamw_state(params, bits=bits) for _ in range(2)]
    for _ in range(2):
        dtp.adamw_step(params, grads, states[0], **HYPER)
        dtp.adamw_step(clean[0], clean[1], states[1], **HYPER)
        grads[0][301] = 0.0           # its square left fp32's range: the moment is infinite, or held as NaN
    assert torch.isfinite(params[0][~bad]).all()
    if bits == 32:
        assert torch.equal(params[0][~bad], clean[0][0][~bad])
    assert torch.isnan(params[0][10])


def test_rounding_is_right_on_average():
    """A million equal elements: the held moments' mean is within six standard deviations of the wanted value, which is a
    part of a step away from both neighbours; so is the mean of bf16 parameters."""
    n = 1 << 20
    for bits in (8,):
        p = [torch.full((n,), 1.0, device=DEV, dtype=BF16)]
        g = [torch.full((n,), 0.3, device=DEV)]
        g[0][::256] = 1.0              # sets each block's scale
        state = dtp.adamw_state(p, bits=bits)
        dtp.adamw_step(p, g, state, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0)
        m, v = dtp.adamw_moments(state)
        few = torch.ones(n, dtype=torch.bool, device=DEV)
        few[::256] = False
        k = int(few.sum())
        for held, want, step in ((m[0], 0.03, 0.03 / 8), (v[0].sqrt(), math.sqrt(0.001) * 0.3, math.sqrt(0.001) * 0.3 / 8),
                                 (p[0].float(), 1.0 - 1e-3, 2.0 ** -8)):
            mean = float(held[few].double().mean())
            assert abs(mean - want) <= 6 * 0.5 * step / math.sqrt(k) + 1e-6 * want, (mean, want)
            assert held[few].unique().numel() == 2
    # a slow average reaches its gradient: 0.999^3000 of the start is left
    p, g = [torch.zeros(n, device=DEV)], [torch.full((n,), 1e-2, device=DEV)]
    state = dtp.adamw_state(p, bits=8)
    dtp.adamw_step(p, [torch.full((n,), 1e-3, device=DEV)], state, lr=0.0, betas=(0.9, 0.999))
    for _ in range(3000):
        dtp.adamw_step(p, g, state, lr=0.0, betas=(0.9, 0.999))
    v = dtp.adamw_moments(state)[1][0]
    # equal elements: each is the largest of its block and held exactly
    assert abs(float(v.mean()) / (1e-4 * (1 - 0.999 ** 3000) + 1e-9 * 0.999 ** 3000) - 1) <= 3001 * 4 * ROUND


def test_rate_on_the_device_and_graphs():
    """A captured step counts its own steps and reads the rate as it is at each replay."""
    params, grads = _tensors([5000, 33], F32, BF16)
    eager = [p.clone() for p in params]
    copies, ecopies = ([torch.zeros_like(p, dtype=BF16) for p in params] for _ in range(2))
    states = [dtp.adamw_state(params, bits=8) for _ in range(2)]
    lr = torch.tensor(1e-3, device=DEV)
    norm = torch.empty((), device=DEV)
    ws, cws = dtp.adamw_workspace(params), dtp.clip_grad_norm_workspace(grads)
    hyper = dict(betas=(0.9, 0.95), weight_decay=0.1, max_norm=0.1)

    def step():
        dtp.clip_grad_norm(grads, math.inf, norm=norm, workspace=cws)
        dtp.adamw_step(params, grads, states[0], lr=lr, norm=norm, copies=copies, workspace=ws, **hyper)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        rate = 1e-3 * (i + 1)
        lr.fill_(rate)
        graph.replay()
        rate = float(lr)
        dtp.adamw_step(eager, grads, states[1], lr=rate, norm=dtp.clip_grad_norm(grads, math.inf), copies=ecopies, **hyper)
        assert all(torch.equal(a, b) for a, b in zip(params + copies, eager + ecopies))
        for g in grads:
            g.mul_(1.5)
    assert int(states[0]["step"]) == 4
    for k in ("m", "v"):
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(states[0][k], states[1][k]))


def test_other_stream_and_some_copies():
    params, grads = _tensors([5000, 33], F32, BF16)
    params.append(torch.randn(64, device=DEV).to(BF16))
    grads.append(torch.randn(64, device=DEV))
    copy = torch.zeros(33, device=DEV, dtype=BF16)
    state = dtp.adamw_state(params)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    dtp.adamw_step(params, grads, state, copies=[None, copy, None], stream=side, **HYPER)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(copy, params[1].to(BF16)) and int(state["step"]) == 1


@pytest.mark.parametrize("betas", [(0.0, 0.0), (0.0, 0.999), (0.95, 0.0)])
def test_betas_of_zero_and_negative_rates(betas):
    params, grads = _tensors([300], F32, F32)
    state = dtp.adamw_state(params)
    before = params[0].clone()
    hyper = dict(lr=-1e-3, betas=betas, eps=1e-6, weight_decay=0.0)
    dtp.adamw_step(params, grads, state, **hyper)
    zero = torch.zeros(300, device=DEV)
    want, _, _, size = _exact(before, grads[0], zero, zero, 1, **hyper)
    assert ((params[0].double() - want).abs() <= 16 * ROUND * (size + 1e-3)).all()


def test_offsets_beyond_32_bits():
    """A tensor of more than 2^32 elements, its ends set: they move as those of small tensors do, and nothing between."""
    n, k = (1 << 32) + 300, 700
    p, g = (torch.zeros(n, dtype=BF16, device=DEV) for _ in range(2))
    state = dtp.adamw_state([p], bits=8)
    gen = torch.Generator(device=DEV).manual_seed(1)
    ends = [torch.randn(k, generator=gen, device=DEV).to(BF16) for _ in range(4)]
    p[:k], p[-k:], g[:k], g[-k:] = ends
    dtp.adamw_step([p], [g], state, **HYPER)
    for before, grad, at in ((ends[0], ends[2], slice(0, k)), (ends[1], ends[3], slice(n - k, n))):
        zero = torch.zeros(k, device=DEV)
        want, em, _, size = _exact(before, grad, zero, zero, 1, **HYPER)
        _check_params(p[at], want, size, before)
        held = state["m"][0][at].float() * state["m_scale"][0].repeat_interleave(256)[: n][at] if at.start == 0 else None
        if held is not None:
            assert ((held.double() - em).abs() <= em.abs() / 8 + 2.0 ** -9 / 448 * em.abs().max()).all()
    assert int(torch.count_nonzero(p[k:-k].view(torch.int16).view(-1))) == 0
    assert float(state["m_scale"][0][-1]) > 0 and float(state["v_scale"][0][1000]) == 0


@pytest.mark.parametrize("std", [1e-2, 1e36])
@pytest.mark.parametrize("limit", [0.0, 1e-300, 1e30])
def test_limits_at_the_ends(std, limit):
    """A limit of zero, or far below fp32's range, leaves the decay alone; norms near fp32's largest are divided by exactly."""
    params, grads = _tensors([3000], F32, F32, std=std)
    norm = dtp.clip_grad_norm(grads, math.inf)
    assert torch.isfinite(norm)
    state = dtp.adamw_state(params)
    before = params[0].clone()
    dtp.adamw_step(params, grads, state, norm=norm, max_norm=limit, **HYPER)
    zero = torch.zeros_like(before)
    want, em, _, size = _exact(before, grads[0], zero, zero, 1, factor=min(1.0, limit / float(norm)), **HYPER)
    if limit < 1.0:
        assert (state["m"][0] == 0).all()
        assert ((params[0].double() - want).abs() <= 16 * ROUND * size + 1e-30).all()
    else:
        assert ((state["m"][0].double() - em).abs() <= 8 * ROUND * em.abs()).all()
