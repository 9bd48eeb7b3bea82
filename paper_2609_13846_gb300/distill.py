"""Running, distilling and tuning a layer whose weights a layout has permuted (Sec. 4).

The part of a layer that a layout permutes, o_proj with the residual and the gated feed-forward block behind its norm,
run forward, differentiated and updated with the library's operators: :func:`dtp.linear`, :func:`dtp.gated_ffn`, their
backward passes and :func:`dtp.clip_grad_norm`.  In :func:`distill_step` the norm between them and the update are plain
torch.  :func:`tune_step` puts the model's end behind the layer, its last norm and its vocabulary, and trains both on the
tokens that follow: :func:`dtp.rms_norm`, :func:`dtp.linear_cross_entropy`, their backward passes and
:func:`dtp.adamw_step`, all of it in one stream's order without a synchronisation, so that a step can be captured.

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


HEAD_NAMES = ("head", "gamma_out")


def head_forward(w: dict, y: torch.Tensor, targets: torch.Tensor):
    """(loss [T] fp32 of each token, 0 where the target is -100, and what :func:`head_backward` needs) of the model's end:
    the norm of y [T, d] with the gain gamma_out [d] fp32, and the vocabulary's rows head [V, d]."""
    h, rms = dtp.rms_norm(y, w["gamma_out"], eps=EPS)
    loss, lse = dtp.linear_cross_entropy(h, w["head"], targets)
    return loss, (y, h, rms, lse, targets)


def head_backward(w: dict, dloss: torch.Tensor, kept) -> tuple[torch.Tensor, dict]:
    """(dy, gradients of head and gamma_out) for dloss [T] fp32."""
    y, h, rms, lse, targets = kept
    dh, dhead = dtp.linear_cross_entropy_backward(dloss, h, w["head"], targets, lse)
    dy, dgamma = dtp.rms_norm_backward(dh, y, w["gamma_out"], rms)
    return dy, dict(head=dhead, gamma_out=dgamma)


def tune_state(master: dict, dtype: torch.dtype = torch.bfloat16, bits: int = 32) -> dict:
    """What :func:`tune_step` keeps between steps for fp32 master weights (o, gate, up, down, gamma, head, gamma_out): their
    copies in ``dtype`` that the layer runs on (bf16, or with fp32 the weights themselves), and the optimiser's states, in
    ``bits`` for the matrices and 32 for the gains."""
    if dtype not in (torch.bfloat16, torch.float32):
        raise TypeError(f"a layer runs in bfloat16 or float32, got {dtype}")
    matrices = [k for k, v in master.items() if v.dim() == 2]
    gains = [k for k, v in master.items() if v.dim() == 1]
    return dict(matrices=matrices, gains=gains, copies={k: master[k].to(dtype) for k in matrices},
                adamw=dtp.adamw_state([master[k] for k in matrices], bits=bits),
                adamw_gains=dtp.adamw_state([master[k] for k in gains]))


def tune_step(master: dict, state: dict, attn: torch.Tensor, x: torch.Tensor, targets: torch.Tensor, lr, max_norm: float,
              betas=(0.9, 0.95), weight_decay: float = 0.1):
    """One AdamW step of the layer and the model's end on the mean loss of the tokens with a target.

    master: fp32 weights, updated in place as ``state`` (of :func:`tune_state`) is; lr a number or a 0-d fp32 tensor on the
    device.  Gradients count clipped to the global norm max_norm; gains are not decayed.  Returns (loss, gradient norm), both 0-d
    tensors; a step whose norm is not finite changes nothing.
    """
    w = dict(state["copies"], **{k: master[k] for k in state["gains"]})
    y, _, kept = layer_forward(w, attn, x, save=True)
    loss, end = head_forward(w, y, targets)
    share = (targets != -100).float()
    share = share / share.sum().clamp(min=1.0)
    dy, grads = head_backward(w, share, end)
    grads.update(layer_backward(w, dy, kept))
    norm = dtp.clip_grad_norm([grads[k] for k in state["matrices"] + state["gains"]], float("inf"))
    common = dict(lr=lr, betas=betas, norm=norm, max_norm=max_norm)
    copies = [state["copies"][k] for k in state["matrices"]]
    copies = [c if c.dtype == torch.bfloat16 else None for c in copies]
    dtp.adamw_step([master[k] for k in state["matrices"]], [grads[k] for k in state["matrices"]], state["adamw"],
                   weight_decay=weight_decay, copies=copies, **common)
    dtp.adamw_step([master[k] for k in state["gains"]], [grads[k] for k in state["gains"]], state["adamw_gains"],
                   weight_decay=0.0, **common)
    return (loss * share).sum(), norm


def make_head(d: int, V: int, seed: int, device="cuda:0") -> dict:
    """A seeded vocabulary and last gain, in fp32."""
    g = torch.Generator(device=device).manual_seed(seed)
    return dict(head=torch.randn((V, d), generator=g, device=device) / d ** 0.5, gamma_out=torch.ones(d, device=device))


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
    # the same layer with the model's end behind it, on the tokens that follow
    master.update(make_head(d, 32000, seed=4))
    targets = torch.randint(0, 32000, (T,), generator=g, device="cuda:0")
    state = tune_state(master, bits=8)
    for i in range(20):
        loss, norm = tune_step(master, state, group, x, targets, lr=1e-3, max_norm=1.0)
        if i % 5 == 0 or i == 19:
            print(f"tokens, step {i}: loss {float(loss):.5f}, gradient norm {float(norm):.4f}")


if __name__ == "__main__":
    main()
