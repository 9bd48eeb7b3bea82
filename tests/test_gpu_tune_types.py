"""distill.tune_step on layers that run in other types than bf16."""
import pytest
import torch

from paper_2609_13846_gb300 import distill

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _model(T, dtype):
    dense, _, attn, x = distill.make_layer(256, 384, 8, 4, 32, T, seed=5, device=DEV)
    master = {k: v.float() for k, v in dense.items()}
    master.update(distill.make_head(256, 700, seed=6, device=DEV))
    g = torch.Generator(device=DEV).manual_seed(7)
    return master, attn.to(dtype), x.to(dtype), torch.randint(0, 700, (T,), generator=g, device=DEV)


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_in_fp32(bits):
    """The layer runs on the fp32 weights themselves: the step is AdamW's of the exact gradient, whose sign each weight follows."""
    master, attn, x, targets = _model(70, torch.float32)
    state = distill.tune_state(master, dtype=torch.float32, bits=bits)
    before = {k: v.clone() for k, v in master.items()}
    p = {k: v.double().requires_grad_() for k, v in before.items()}

    def norm(r, gamma):
        return r * torch.rsqrt(r.square().mean(-1, keepdim=True) + distill.EPS) * gamma

    r = x.double() + attn.double() @ p["o"].t()
    h = norm(r, p["gamma"])
    out = r + (torch.nn.functional.silu(h @ p["gate"].t()) * (h @ p["up"].t())) @ p["down"].t()
    want = torch.nn.functional.cross_entropy(norm(out, p["gamma_out"]) @ p["head"].t(), targets)
    ref = dict(zip(p, torch.autograd.grad(want, list(p.values()))))
    want = float(want.detach())
    for i in range(2):
        loss, n = distill.tune_step(master, state, attn, x, targets, lr=1e-3, max_norm=0.5)
        if i:
            continue
        # a dozen products of fp32 sums of some hundred terms, 2^-24 each
        assert abs(float(loss) - want) <= 1e-5 * want
        total = float(torch.stack([g.square().sum() for g in ref.values()]).sum().sqrt())
        assert abs(float(n) - total) <= 1e-4 * total
        for k, v in master.items():
            decay = 0.1 if v.dim() == 2 else 0.0
            moved = (v.double() - before[k].double() * (1 - 1e-3 * decay)) / 1e-3
            assert (moved.abs() <= 1.0 + 1e-3).all(), k
            big = ref[k].abs() > 1e-2 * ref[k].norm() / ref[k].numel() ** 0.5
            assert (torch.sign(moved[big]) == -torch.sign(ref[k][big])).all(), k
    assert int(state["adamw"]["step"]) == 2


def test_types_without_a_layer_are_refused():
    master, _, _, _ = _model(2, torch.float32)
    for dtype in (torch.float16, torch.float64):
        with pytest.raises(TypeError, match="bfloat16 or float32"):
            distill.tune_state(master, dtype=dtype)
