"""Running and distilling a layer whose weights a layout has permuted (Sec. 4).

The part of a layer that a layout permutes, o_proj with the residual and the gated feed-forward block behind its norm,
run forward, differentiated and updated with the library's operators: :func:`dtp.linear`, :func:`dtp.gated_ffn`, their
backward passes and :func:`dtp.clip_grad_norm`.  The norm between them and the optimiser's update are plain torch.

    python -m paper_2609_13846_gb300.distill        # a perturbed, permuted layer learns its dense teacher's output
"""
from __future__ import annotations

import torch

from . import dtp, synth

EPS = 1e-6
NAMES = ("o", "gate", "up", "down", "gamma")


def _norm(r: torch.Tensor, gamma: torch.Tensor):
    """(gamma * r / rms in r's dtype, r / rms in fp32, rms [T] fp32)."""
    f = r.float()
    rms = (f.square().mean(-1) + EPS).sqrt()
    n = f / rms[:, None]
    return (n * gamma).to(r.dtype), n, rms


def layer_forward(w: dict, attn: torch.Tensor, x: torch.Tensor, save: bool = False):
    """Y = r + FFN(norm(r)) with r = x + attn W_o^T, and the rms of r (what the affinity scores take as ``rms``).

    w: o [d, Hq*hd], gate and up [N, d], down [d, N] in attn's dtype, gamma [d] fp32; attn [T, Hq*hd] the heads'
    outputs, x [T, d] the residual stream.  With ``save`` a third value holds what :func:`layer_backward` needs.
    """
    r = dtp.linear(attn, w["o"], residual=x)
    h, n, rms = _norm(r, w["gamma"])
    y = dtp.gated_ffn(h, w["gate"], w["up"], w["down"], residual=r, save=save)
    if not save:
        return y, rms
    y, saved = y
    return y, rms, (attn, h, n, rms, saved)


def layer_backward(w: dict, dy: torch.Tensor, kept) -> dict:
    """Gradients of the layer's weights (those of o, gate, up and down in their dtype, gamma's in fp32) and of attn
    and x, for dy [T, d]."""
    attn, h, n, rms, saved = kept
    dh, dgate, dup, ddown = dtp.gated_ffn_backward(dy, h, w["gate"], w["up"], w["down"], saved)
    dn = dh.float() * w["gamma"]
    dr = dy.float() + (dn - n * (dn * n).mean(-1, keepdim=True)) / rms[:, None]
    dr = dr.to(dy.dtype)
    dattn, do, _ = dtp.linear_backward(dr, attn, w["o"])
    return dict(o=do, gate=dgate, up=dup, down=ddown, gamma=(dh.float() * n).sum(0), attn=dattn, x=dr)


def distill_step(master: dict, teacher: torch.Tensor, attn: torch.Tensor, x: torch.Tensor, lr: float, max_norm: float):
    """One step of gradient descent on |Y - teacher|^2 / 2T, gradients clipped by their global norm.

    master: the student's weights in fp32, updated in place; the layer runs on their copies in attn's dtype.  Returns
    (loss, gradient norm), both 0-d tensors; a step whose norm is not finite changes nothing.
    """
    w = {k: v if k == "gamma" else v.to(attn.dtype) for k, v in master.items()}
    y, _, kept = layer_forward(w, attn, x, save=True)
    diff = y.float() - teacher.float()
    loss = diff.square().sum() / (2 * x.shape[0])
    grads = layer_backward(w, (diff / x.shape[0]).to(y.dtype), kept)
    grads = [grads[k] for k in NAMES]
    norm = dtp.clip_grad_norm(grads, max_norm)
    step = torch.where(torch.isfinite(norm), lr, 0.0)
    for k, g in zip(NAMES, grads):
        master[k] -= step * torch.nan_to_num(g.float(), 0.0, 0.0, 0.0)
    return loss, norm


def make_layer(d: int, N: int, Hq: int, G: int, head_dim: int, T: int, seed: int, device="cuda:0"):
    """(dense bf16 weights, attn, x) of one seeded layer."""
    P = synth.make_attention_inputs(T, d, Hq, head_dim, seed, device=device)
    W = synth.make_dense_weights(1, d, Hq, G, head_dim, N, seed + 1, device=device)
    x = torch.randn((T, d), generator=torch.Generator(device=device).manual_seed(seed + 2), device=device)
    dense = dict(o=W["o"][0], gate=W["gate"][0], up=W["up"][0], down=W["down"][0], gamma=P["gamma"])
    return dense, W, P["attn"], x.to(torch.bfloat16)


def main():
    d, N, Hq, G, hd, T, D = 1024, 3072, 16, 8, 128, 4096, 4
    dense, W, attn, x = make_layer(d, N, Hq, G, hd, T, seed=1)
    teacher, _ = layer_forward(dense, attn, x)
    # a layout from the weights' scores; the permuted layer computes the same function
    A = dtp.affinity_accumulate(x, synth.make_layer(d, G, N, T, 3, device="cuda:0")["C"], dense["gate"], dense["up"])
    lay = dtp.search_layout(A, D=D, iters=10)
    perm, heads, _ = dtp.apply_layout(W, lay["h"][None], lay["nu"][None], D=D, head_dim=hd)
    group = attn.view(T, G, -1)[:, heads[0].long()].reshape(T, -1).contiguous()
    student = dict(o=perm["o"][0], gate=perm["gate"][0], up=perm["up"][0], down=perm["down"][0], gamma=dense["gamma"])
    y, _ = layer_forward(student, group, x)
    print(f"permuted layer: largest difference {float((y.float() - teacher.float()).abs().max()):.3g}")
    g = torch.Generator(device="cuda:0").manual_seed(9)
    master = {k: v.float() + 0.1 * float(v.float().std()) * torch.randn(v.shape, generator=g, device=v.device)
              for k, v in student.items()}
    for i in range(20):
        loss, norm = distill_step(master, teacher, group, x, lr=2e-2, max_norm=5.0)
        if i % 5 == 0 or i == 19:
            print(f"step {i}: loss {float(loss):.5f}, gradient norm {float(norm):.4f}")


if __name__ == "__main__":
    main()
