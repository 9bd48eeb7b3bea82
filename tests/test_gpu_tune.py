"""The norm, the vocabulary's loss, the clipping and the update together, as a training step uses them."""
import pytest
import torch

from paper_2609_13846_gb300 import distill, dtp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
V = 700


def _model(T=300, dtype=torch.bfloat16):
    dense, _, attn, x = distill.make_layer(256, 384, 8, 4, 32, T, seed=5, device=DEV)
    master = {k: v.float() for k, v in dense.items()}
    master.update(distill.make_head(256, V, seed=6, device=DEV))
    g = torch.Generator(device=DEV).manual_seed(7)
    targets = torch.randint(0, V, (T,), generator=g, device=DEV)
    targets[::7] = -100
    return master, attn.to(dtype), x.to(dtype), targets


def _reference(master, copies, attn, x, targets):
    """(loss, gradients) of torch's autograd in fp64 on the weights that the layer runs on."""
    p = {k: copies.get(k, v).double().requires_grad_() for k, v in master.items()}

    def norm(r, gamma):
        return r * torch.rsqrt(r.square().mean(-1, keepdim=True) + distill.EPS) * gamma

    r = x.double() + attn.double() @ p["o"].t()
    h = norm(r, p["gamma"])
    y = r + (torch.nn.functional.silu(h @ p["gate"].t()) * (h @ p["up"].t())) @ p["down"].t()
    z = norm(y, p["gamma_out"]) @ p["head"].t()
    loss = torch.nn.functional.cross_entropy(z, targets)
    return loss.detach(), dict(zip(p, torch.autograd.grad(loss, list(p.values()))))


@pytest.mark.parametrize("T", [1, 64, 300])
def test_gradients_are_autograds(T):
    """bf16: the path rounds r, h, H, y, the last h, dZ, its dh, dG, dU, dr and each gradient once (2^-8 sqrt(1/5) of a value on
    average); 12 roundings in quadrature are below 1.3% of a gradient's norm."""
    master, attn, x, targets = _model(T)
    if T == 1:
        targets[0] = 3
    w = {k: v.to(torch.bfloat16) if v.dim() == 2 else v for k, v in master.items()}
    y, _, kept = distill.layer_forward(w, attn, x, save=True)
    loss, end = distill.head_forward(w, y, targets)
    share = (targets != -100).float()
    share /= share.sum()
    dy, grads = distill.head_backward(w, share, end)
    grads.update(distill.layer_backward(w, dy, kept))
    want, ref = _reference(master, {k: v for k, v in w.items() if v.dim() == 2}, attn, x, targets)
    assert abs(float((loss * share).sum()) - float(want)) <= 2.0 ** -8 * float(want)
    for k, g in ref.items():
        assert (grads[k].double() - g).norm() <= 1.3e-2 * g.norm(), k


@pytest.mark.parametrize("bits", [32, 8])
def test_step_updates_what_it_says(bits):
    """The master weights move by AdamW's first step of the clipped gradient: at most lr / (1 - eps') each beside the decay, in the
    direction of the gradient's sign wherever that is far above the gradient's error; the copies are theirs, rounded."""
    master, attn, x, targets = _model()
    state = distill.tune_state(master, bits=bits)
    before = {k: v.clone() for k, v in master.items()}
    _, ref = _reference(master, state["copies"], attn, x, targets)
    loss, norm = distill.tune_step(master, state, attn, x, targets, lr=1e-3, max_norm=0.5)
    total = float(torch.stack([g.square().sum() for g in ref.values()]).sum().sqrt())
    assert abs(float(norm) - total) <= 2e-2 * total
    for k, v in master.items():
        decay = 0.1 if v.dim() == 2 else 0.0
        moved = (v.double() - before[k].double() * (1 - 1e-3 * decay)) / 1e-3
        assert (moved.abs() <= 1.0 + 1e-3).all(), k
        big = ref[k].abs() > ref[k].norm() / ref[k].numel() ** 0.5       # above the root mean square: off by less than themselves
        assert (torch.sign(moved[big]) == -torch.sign(ref[k][big])).float().mean() > 0.99, k
        if v.dim() == 2:
            assert torch.equal(state["copies"][k], v.to(torch.bfloat16))
    assert int(state["adamw"]["step"]) == int(state["adamw_gains"]["step"]) == 1


def test_captured_steps_are_the_eager_ones():
    """A captured step, replayed with other inputs and another rate, gives the eager steps' weights bit for bit."""
    master, attn, x, targets = _model()
    eager = {k: v.clone() for k, v in master.items()}
    states = [distill.tune_state(m, bits=8) for m in (master, eager)]
    lr = torch.tensor(1e-3, device=DEV)
    inputs = [attn.clone(), x.clone(), targets.clone()]
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        loss, norm = distill.tune_step(master, states[0], *inputs, lr=lr, max_norm=0.5)
    for i in range(3):
        for a, b in zip(inputs, (attn, x, targets)):
            a.copy_(b.roll(i, 0))
        lr.fill_(1e-3 / (i + 1))
        graph.replay()
        want, wnorm = distill.tune_step(eager, states[1], *[t.clone() for t in inputs], lr=float(lr), max_norm=0.5)
        assert torch.equal(loss, want) and torch.equal(norm, wnorm)
        assert all(torch.equal(master[k], eager[k]) for k in master), i


def test_a_step_with_a_bad_token_changes_nothing():
    """Infinite hidden states make the norm infinite or NaN: nothing moves, and the next step does."""
    master, attn, x, targets = _model()
    state = distill.tune_state(master)
    before = {k: v.clone() for k, v in master.items()}
    bad = x.clone()
    bad[1, 3] = float("inf")
    assert targets[1] != -100
    _, norm = distill.tune_step(master, state, attn, bad, targets, lr=1e-3, max_norm=1.0)
    assert not torch.isfinite(norm)
    assert all(torch.equal(v, before[k]) for k, v in master.items()) and int(state["adamw"]["step"]) == 0
    distill.tune_step(master, state, attn, x, targets, lr=1e-3, max_norm=1.0)
    assert int(state["adamw"]["step"]) == 1 and not torch.equal(master["head"], before["head"])


def test_the_norms_rms_is_the_producers():
    """dtp.rms_norm's second result is what the affinity's producer takes."""
    g = torch.Generator(device=DEV).manual_seed(1)
    r = torch.randn((130, 256), generator=g, device=DEV).to(torch.bfloat16)
    attn = torch.randn((130, 512), generator=g, device=DEV).to(torch.bfloat16)
    W_o = (torch.randn((256, 512), generator=g, device=DEV) * 0.02).to(torch.bfloat16)
    gamma = torch.ones(256, device=DEV)
    _, rms = dtp.rms_norm(r, gamma, eps=distill.EPS)
    C = dtp.head_writes(attn, W_o, gamma, rms, head_dim=32)
    want = torch.einsum("thk,dhk->htd", attn.double().view(130, 16, 32), W_o.double().view(256, 16, 32))
    want = want / (r.double().square().mean(-1) + distill.EPS).sqrt()[None, :, None]
    assert (C.double() - want).norm() <= 2.0 ** -8 * want.norm()
