"""Calls that write a caller's tensors tell autograd so: a graph that saved one must not differentiate with its new values."""
import pytest
import torch

from paper_2609_13846_gb300 import dtp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


def _refuses_backward(saved, write):
    a = torch.ones_like(saved, requires_grad=True)
    loss = (a * saved).sum()           # saves it for a's gradient
    write()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_updated_weights_and_copies():
    p = [torch.randn(300, device=DEV), torch.randn(70, device=DEV)]
    grads, copies = [t.to(BF16) for t in p], [torch.zeros(300, dtype=BF16, device=DEV), None]
    state = dtp.adamw_state(p, bits=8)
    step = lambda: dtp.adamw_step(p, grads, state, lr=1e-3, copies=copies)  # noqa: E731
    for t in (*p, copies[0], state["m"][0], state["v_scale"][1], state["step"]):
        before = t._version
        step()
        assert t._version > before
    _refuses_backward(p[1], step)
    _refuses_backward(copies[0], step)
    held = [g._version for g in grads]
    step()
    assert [g._version for g in grads] == held
    weight = torch.nn.Parameter(torch.randn(40, device=DEV))
    dtp.adamw_step([weight], [torch.ones(40, device=DEV)], dtp.adamw_state([weight]), lr=1e-3)
    before = p[0]._version
    with pytest.raises(dtp.DTPError):
        dtp.adamw_step(p, grads, state, lr=1e-3, betas=(1.0, 0.9))
    assert p[0]._version == before


def test_results_in_given_tensors():
    x, gamma = torch.randn((5, 64), device=DEV), torch.ones(64, device=DEV)
    y = torch.zeros_like(x)
    _refuses_backward(y, lambda: dtp.rms_norm(x, gamma, Y=y))
    _refuses_backward(x, lambda: dtp.rms_norm(x, gamma, Y=x))
    w = torch.randn((64, 64), device=DEV)
    _refuses_backward(y, lambda: dtp.linear(x, w, Y=y))
    _refuses_backward(y, lambda: dtp.gated_ffn(x, w, w, w, Y=y))
    g = [torch.randn(100, device=DEV), torch.randn(33, device=DEV)]
    out = [torch.zeros_like(t) for t in g]
    _refuses_backward(g[1], lambda: dtp.clip_grad_norm(g, 1.0))
    _refuses_backward(out[0], lambda: dtp.clip_grad_norm(g, 1.0, out=out))


def test_tensors_without_versions():
    with torch.inference_mode():
        p, x = torch.randn(40, device=DEV), torch.randn((3, 64), device=DEV)
        state = dtp.adamw_state([p])
        before = p.clone()
        dtp.adamw_step([p], [torch.ones(40, device=DEV)], state, lr=1e-3)
        dtp.rms_norm(x, torch.ones(64, device=DEV), Y=x)
    dtp.adamw_step([p], [torch.ones(40, device=DEV)], state, lr=1e-3)
    assert not torch.equal(p, before) and int(state["step"]) == 2
