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


def test_two_streams_at_once():
    """Calls of two streams with workspaces of their own, in flight together, give what they give one after the other."""
    def work(seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        x = torch.randn((600 + seed, 256), generator=g, device=DEV).to(torch.bfloat16)
        w = (torch.randn((9000, 256), generator=g, device=DEV) * 0.1).to(torch.bfloat16)
        y = torch.randint(0, 9000, (x.shape[0],), generator=g, device=DEV)
        y[::5] = -100
        p = [torch.randn(n, generator=g, device=DEV) for n in (100_000, 33)]
        gr = [torch.randn(n, generator=g, device=DEV).to(torch.bfloat16) for n in (100_000, 33)]
        gamma = torch.rand(256, generator=g, device=DEV) + 0.5
        dl = torch.full((x.shape[0],), 1e-3, device=DEV)
        state = dtp.adamw_state(p, bits=8)
        return x, w, y, p, gr, gamma, dl, state

    def run(x, w, y, p, gr, gamma, dl, state):
        out = []
        for _ in range(3):
            h, rms = dtp.rms_norm(x, gamma)
            loss, lse = dtp.linear_cross_entropy(h, w, y)
            dh, dw = dtp.linear_cross_entropy_backward(dl, h, w, y, lse)
            dx, dgamma = dtp.rms_norm_backward(dh, x, gamma, rms)
            dtp.adamw_step(p, gr, state, lr=1e-3)
            out = [h, loss, lse, dw, dx, dgamma]
        return out + p + state["m_scale"] + state["v_scale"]

    want = [run(*work(s)) for s in (1, 2)]
    inputs, streams, got = [work(s) for s in (1, 2)], [torch.cuda.Stream() for _ in range(2)], []
    torch.cuda.synchronize()
    for a, s in zip(inputs, streams):
        with torch.cuda.stream(s):
            got.append(run(*a))
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_compaction_of_more_than_a_run_of_tokens():
    """dX alone of more than 2^18 tokens, half of them padding: each token's row at its own place."""
    T, d, V = (1 << 18) + 4097, 64, 200
    g = torch.Generator(device=DEV).manual_seed(11)
    x = torch.randn((T, d), generator=g, device=DEV).to(torch.bfloat16)
    w = (torch.randn((V, d), generator=g, device=DEV) * 0.2).to(torch.bfloat16)
    y = torch.randint(0, V, (T,), generator=g, device=DEV)
    y[torch.rand(T, generator=g, device=DEV) < 0.5] = -100
    _, lse = dtp.linear_cross_entropy(x, w, y)
    dl = torch.rand(T, generator=g, device=DEV)
    dx = torch.empty_like(x)
    ws = dtp.linear_cross_entropy_workspace(T, d, V, torch.bfloat16, DEV, backward=True)
    st = dtp.lib().dtp_linear_cross_entropy_backward(dl.data_ptr(), x.data_ptr(), w.data_ptr(), y.data_ptr(), lse.data_ptr(), T, d, V, -100,
                                                     dtp.DTP_BF16, dx.data_ptr(), None, ws.data_ptr(), ws.numel(),
                                                     torch.cuda.current_stream().cuda_stream)
    assert st == dtp.DTP_OK
    live = y != -100
    dz = torch.softmax(x.double() @ w.double().t(), 1)
    dz.scatter_add_(1, torch.where(live, y, 0)[:, None], -torch.ones((T, 1), dtype=torch.float64, device=DEV))
    dz *= (dl * live).double()[:, None]
    half = torch.finfo(torch.bfloat16).eps / 2
    ref = dz @ w.double()
    # dX is rounded once, each element of dZ once (1.01: the second order); 2^-12 is far above what fp32 logits and sums of 200 add
    assert ((dx.double() - ref).abs() <= half * ref.abs() + (1.01 * half + 2.0 ** -12) * dz.abs() @ w.double().abs()).all()
    assert (dx[~live] == 0).all()
