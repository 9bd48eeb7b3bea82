"""The measured cases of the training and serving operators: a linear layer with its epilogue, the gated
feed-forward block, and the clipped gradient of many tensors.

After a layout has been applied to a model, the model's layers are run (calibration again, serving) and
distilled: every token batch goes through o_proj with the residual added and through the gated block, forward
and backward, and each step's gradients are clipped by their global norm.  Each listed case is one such call
(a training case: forward and backward) at sizes of the repository's workloads, tests and benchmark, or generic
odd ones; ``draw`` spreads the same calls over the whole range of sizes.

A case is a dict with the operator ``op`` ("linear", "ffn" or "clip") and its sizes:
  linear: T tokens, K inputs, N outputs, act, bias, residual, train, dtype
  ffn:    T tokens, d model width, N neurons, act, residual, train, dtype
  clip:   tensors, total (elements, about), f32_share (of the tensors in fp32, the others bf16), tight (packed without
          alignment), ratio (norm over the limit; below 1 nothing is clipped), inplace, shape_seed; layers > 0 gives the
          tensors of so many transformer layers instead (d, N and heads of the 1024-wide workload)
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
ACTS = ("none", "silu", "gelu", "relu")


def listed():
    return [
        # serving: one token through o_proj of the 4096-wide workload, residual added
        dict(name="o_proj_token", op="linear", dtype="bf16", T=1, K=4096, N=4096, act="none", bias=False, residual=True,
             train=False),
        # a prompt of odd length through o_proj of the 1024-wide workload (16 heads of 128)
        dict(name="o_proj_prompt", op="linear", dtype="bf16", T=1003, K=2048, N=1024, act="none", bias=False,
             residual=True, train=False),
        # an fp32 layer with every part of the epilogue, odd sizes: the tight-check mode
        dict(name="linear_f32_odd", op="linear", dtype="f32", T=515, K=1536, N=1001, act="gelu", bias=True,
             residual=True, train=False),
        # training step of a wide layer with bias and activation
        dict(name="linear_train", op="linear", dtype="bf16", T=8192, K=1024, N=4096, act="silu", bias=True,
             residual=False, train=True),
        # serving: one token through the block of the 1024-wide workload
        dict(name="ffn_token", op="ffn", dtype="bf16", T=1, d=1024, N=3072, act="silu", residual=True, train=False),
        # serving: a batch of single tokens through the widest workload's block
        dict(name="ffn_batch32", op="ffn", dtype="bf16", T=32, d=4096, N=14336, act="silu", residual=True, train=False),
        # the benchmark's token batch through its layer
        dict(name="ffn_prompt", op="ffn", dtype="bf16", T=16384, d=1024, N=3072, act="silu", residual=True, train=False),
        # a distillation step of the widest block
        dict(name="ffn_train", op="ffn", dtype="bf16", T=4096, d=4096, N=14336, act="silu", residual=True, train=True),
        # fp32 training step at odd sizes: the tight-check mode
        dict(name="ffn_train_f32_odd", op="ffn", dtype="f32", T=257, d=520, N=1001, act="gelu", residual=False,
             train=True),
        # the gradients of one layer, out of place, over the limit
        dict(name="clip_layer", op="clip", layers=1, tensors=0, total=0, f32_share=0.0, tight=False, ratio=3.7,
             inplace=False, shape_seed=0),
        # the gradients of a 28-layer model, out of place, over the limit
        dict(name="clip_model", op="clip", layers=28, tensors=0, total=0, f32_share=0.0, tight=False, ratio=3.7,
             inplace=False, shape_seed=0),
        # many odd tensors of both types packed without alignment, in place, under the limit
        dict(name="clip_mixed", op="clip", layers=0, tensors=301, total=60_000_000, f32_share=0.5, tight=True, ratio=0.5,
             inplace=True, shape_seed=7),
    ]


# ------------------------------------------------------------------------ draws --

MOST_FLOPS = 4.3e12
MOST_ELEMENTS = 440_000_000


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A layer's width: a common one, any multiple of 8, or any number."""
    kind = rng.random()
    if kind < 0.4:
        return rng.choice([w for w in (64, 768, 1024, 1536, 2048, 4096, 8192, 14336) if lo <= w <= hi])
    w = _log(rng, lo, hi)
    return max(8, w // 8 * 8) if kind < 0.8 else w


def draw(rng):
    op = rng.choice(["linear", "linear", "ffn", "ffn", "ffn", "clip", "clip"])
    if op == "clip":
        total = _log(rng, 2000, MOST_ELEMENTS)
        return dict(op="clip", layers=0, tensors=min(_log(rng, 1, 400), total), total=total,
                    f32_share=rng.choice([0.0, 0.0, 0.5, 1.0]), tight=rng.random() < 0.5,
                    ratio=rng.choice([0.5, 1.5, 3.7, 90.0]), inplace=False, shape_seed=rng.randrange(1 << 20))
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    train = rng.random() < 0.4
    c = dict(op=op, dtype=dtype, T=_log(rng, 1, 16384))
    if op == "linear":
        c.update(K=_width(rng, 64, 8192), N=_width(rng, 64, 14336), act=rng.choice(ACTS), bias=rng.random() < 0.5,
                 residual=rng.random() < 0.5, train=train)
    else:
        c.update(d=_width(rng, 64, 4096), N=_width(rng, 96, 14336), act=rng.choice(["silu", "silu", "gelu"]),
                 residual=rng.random() < 0.7, train=train)
    most = MOST_FLOPS if dtype == "bf16" else MOST_FLOPS / 8
    while work(c)["flops"] > most:
        c["T"] = c["T"] * 2 // 3
    return c


# ------------------------------------------------------------------------- work --

def _e(c):
    return 2 if c["dtype"] == "bf16" else 4


def work(c):
    if c["op"] == "clip":
        sizes = _clip_sizes(c)
        each = sum(n * (4 if f32 else 2) for n, f32 in sizes)
        writes = not (c["inplace"] and c["ratio"] <= 1.0)
        return dict(bytes=each * (2 if writes else 1) + 4, flops=(3 if writes else 2) * sum(n for n, _ in sizes))
    T, N, e = c["T"], c["N"], _e(c)
    if c["op"] == "linear":
        K = c["K"]
        values = T * K + N * K + N * c["bias"] + T * N * c["residual"] + T * N
        flops = 2 * T * K * N
        if c["train"]:
            values += T * N + T * K + N * K + N * c["bias"]     # dY; dX, dW, db
            flops += 4 * T * K * N
        return dict(bytes=values * e, flops=flops)
    d = c["d"]
    values = T * d + 3 * N * d + T * d * c["residual"] + T * d
    flops = 6 * T * d * N
    if c["train"]:
        values += T * d + T * d + 3 * N * d                     # dY; dX, dW_gate, dW_up, dW_down
        flops += 12 * T * d * N
    return dict(bytes=values * e, flops=flops)


# ----------------------------------------------------------------------- inputs --

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, std, dtype):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).mul_(std).to(dtype)


def _tokens(g, T, d, dtype):
    """Normalised layer inputs: N(0,1) with 4 outlier channels scaled by 20, as in the calibration workloads."""
    x = torch.randn((T, d), generator=g, device=DEV, dtype=torch.float32)
    x[:, torch.randperm(d, generator=g, device=DEV)[:4]] *= 20.0
    return x.to(dtype)


def _clip_sizes(c):
    """[(elements, in fp32)] of the case's tensors."""
    if c["layers"]:
        d, N, q, kv = 1024, 3072, 2048, 1024
        layer = [q * d, kv * d, kv * d, d * q, N * d, N * d, d * N, d, d, 128, 128]
        return [(n, False) for _ in range(c["layers"]) for n in layer]
    r = random.Random(c["shape_seed"])
    w = [math.exp(r.gauss(0.0, 2.0)) for _ in range(c["tensors"])]
    s = sum(w)
    return [(max(1, int(c["total"] * x / s)), r.random() < c["f32_share"]) for x in w]


def prepare(c, seed):
    g = _gen(seed)
    if c["op"] == "clip":
        return _prepare_clip(c, g)
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    T, N = c["T"], c["N"]
    s = dict(case=c)
    if c["op"] == "linear":
        K = c["K"]
        s.update(X=_tokens(g, T, K, dt), W=_normal(g, (N, K), 0.02, dt), bias=None, residual=None)
        if c["bias"]:
            s["bias"] = _normal(g, (N,), 0.5, dt)
        out = N
    else:
        d = c["d"]
        s.update(X=_tokens(g, T, d, dt), W_gate=_normal(g, (N, d), 0.02, dt), W_up=_normal(g, (N, d), 0.02, dt),
                 W_down=_normal(g, (d, N), 0.02, dt), residual=None)
        out = d
    if c["residual"]:
        s["residual"] = _normal(g, (T, out), 1.0, dt)
    if c["train"]:
        s["dY"] = _normal(g, (T, out), 1e-2, dt)
    if own:         # the workspace that a serving or training loop keeps
        from paper_2609_13846_gb300 import dtp
        if c["op"] == "linear":
            s["workspace"] = dtp.linear_workspace(T, c["K"], N, s["X"].dtype, DEV, backward=c["train"])
        else:
            s["workspace"] = dtp.gated_ffn_workspace(T, c["d"], N, s["X"].dtype, DEV, backward=c["train"])
    return s


def _prepare_clip(c, g):
    sizes = _clip_sizes(c)
    flat, views = {}, []
    offsets, used = [], {False: 0, True: 0}
    for n, f32 in sizes:
        offsets.append(used[f32])
        used[f32] += n if c["tight"] else (n + 63) // 64 * 64
    for f32, n in used.items():
        if n:
            flat[f32] = torch.zeros(n, device=DEV, dtype=torch.float32 if f32 else torch.bfloat16)
    for (n, f32), at in zip(sizes, offsets):
        v = flat[f32][at:at + n]
        # gradients of layers differ in scale by orders of magnitude
        v.copy_(torch.randn((n,), generator=g, device=DEV).mul_(10.0 ** -(1 + len(views) % 4)))
        views.append(v)
    norm = math.sqrt(sum(float(v.double().square().sum()) for v in flat.values()))
    s = dict(case=c, grads=views, flat=[flat[k] for k in sorted(flat)], limit=float(norm / c["ratio"]), out=None)
    if not c["inplace"]:
        dst = {k: torch.zeros_like(v) for k, v in flat.items()}
        s["out"] = [dst[f32][at:at + n] for (n, f32), at in zip(sizes, offsets)]
        s["flat_out"] = [dst[k] for k in sorted(dst)]
    if own:
        from paper_2609_13846_gb300 import dtp
        s["workspace"] = dtp.clip_grad_norm_workspace(views)
    return s


# ------------------------------------------------------------------ plain forms --

def _act(name, z):
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    return z


def _act_grad(name, z):
    if name == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    if name == "relu":
        return (z > 0).to(z.dtype)
    return torch.ones_like(z)


def _plain_linear(s):
    c, dt = s["case"], s["X"].dtype
    x, w = s["X"].float(), s["W"].float()
    z = x @ w.t()
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y = _act(c["act"], z)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out = dict(Y=y.to(dt))
    if c["train"]:
        dz = s["dY"].float() * _act_grad(c["act"], z)
        out.update(dX=(dz @ w).to(dt), dW=(dz.t() @ x).to(dt))
        if s["bias"] is not None:
            out["dbias"] = dz.sum(0).to(dt)
    return out


def _plain_ffn(s):
    c, dt = s["case"], s["X"].dtype
    x, wg, wu, wd = s["X"].float(), s["W_gate"].float(), s["W_up"].float(), s["W_down"].float()
    g, u = x @ wg.t(), x @ wu.t()
    a = _act(c["act"], g)
    h = a * u
    y = h @ wd.t()
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out = dict(Y=y.to(dt))
    if c["train"]:
        dy = s["dY"].float()
        dh = dy @ wd
        du = dh * a
        dg = dh * u * _act_grad(c["act"], g)
        out.update(dX=(dg @ wg + du @ wu).to(dt), dW_gate=(dg.t() @ x).to(dt), dW_up=(du.t() @ x).to(dt),
                   dW_down=(dy.t() @ h).to(dt))
    return out


def _plain_clip(s):
    squares = [v.float().square().sum() for v in s["grads"]]
    norm = torch.stack(squares).sum().sqrt()
    coef = torch.clamp(s["limit"] / norm, max=1.0)
    out = s["grads"] if s["out"] is None else s["out"]
    [o.copy_(v.float() * coef) for v, o in zip(s["grads"], out)]
    return dict(norm=norm, grads=s["flat"] if s["out"] is None else s["flat_out"])


# ------------------------------------------------------------------- the passes --

def run(s):
    c = s["case"]
    if not own:
        return dict(linear=_plain_linear, ffn=_plain_ffn, clip=_plain_clip)[c["op"]](s)
    from paper_2609_13846_gb300 import dtp
    if c["op"] == "clip":
        norm = dtp.clip_grad_norm(s["grads"], s["limit"], out=s["out"], workspace=s["workspace"])
        return dict(norm=norm, grads=s["flat"] if s["out"] is None else s["flat_out"])
    ws, act = s["workspace"], c["act"]
    if c["op"] == "linear":
        if not c["train"]:
            return dict(Y=dtp.linear(s["X"], s["W"], s["bias"], s["residual"], activation=act, workspace=ws))
        y, z = dtp.linear(s["X"], s["W"], s["bias"], s["residual"], activation=act, save=True, workspace=ws)
        dx, dw, db = dtp.linear_backward(s["dY"], s["X"], s["W"], z, activation=act, bias=s["bias"] is not None,
                                         workspace=ws)
        out = dict(Y=y, dX=dx, dW=dw)
        if db is not None:
            out["dbias"] = db
        return out
    if not c["train"]:
        return dict(Y=dtp.gated_ffn(s["X"], s["W_gate"], s["W_up"], s["W_down"], s["residual"], activation=act,
                                    workspace=ws))
    y, saved = dtp.gated_ffn(s["X"], s["W_gate"], s["W_up"], s["W_down"], s["residual"], activation=act, save=True,
                             workspace=ws)
    dx, dg, du, dd = dtp.gated_ffn_backward(s["dY"], s["X"], s["W_gate"], s["W_up"], s["W_down"], saved,
                                            activation=act, workspace=ws)
    return dict(Y=y, dX=dx, dW_gate=dg, dW_up=du, dW_down=dd)


# ---------------------------------------------------------------- exact results --

EXACT_FLOPS = 6e12      # about 10 s of fp64 on the GPU


def exact(c, seed):
    """The definition in 64 bits: forward values written out, gradients by differentiating the scalar <Y, dY>."""
    if c["op"] != "clip" and work(c)["flops"] > EXACT_FLOPS:
        return None
    s = prepare(c, seed)
    if c["op"] == "clip":
        total = sum(float((v.to(torch.float64) ** 2).sum()) for v in s["flat"])
        norm = math.sqrt(total)
        scale = 1.0 if norm <= s["limit"] else s["limit"] / norm
        return dict(norm=torch.tensor(norm, dtype=torch.float64), grads=[v.to(torch.float64) * scale for v in s["flat"]])
    names = [k for k in ("X", "W", "bias", "W_gate", "W_up", "W_down") if s.get(k) is not None]
    p = {k: s[k].to(torch.float64).requires_grad_(c["train"]) for k in names}
    gates = dict(none=lambda v: v, silu=lambda v: v * torch.sigmoid(v),
                 gelu=lambda v: v * torch.special.ndtr(v), relu=lambda v: v.clamp(min=0))
    f = gates[c["act"]]
    if c["op"] == "linear":
        z = torch.einsum("tk,nk->tn", p["X"], p["W"])
        y = f(z + p["bias"]) if "bias" in p else f(z)
    else:
        h = f(torch.einsum("td,nd->tn", p["X"], p["W_gate"])) * torch.einsum("td,nd->tn", p["X"], p["W_up"])
        y = torch.einsum("tn,dn->td", h, p["W_down"])
    if s["residual"] is not None:
        y = y + s["residual"].to(torch.float64)
    out = dict(Y=y.detach())
    if c["train"]:
        grads = torch.autograd.grad(y, [p[k] for k in names], grad_outputs=s["dY"].to(torch.float64))
        out.update({"d" + k: g for k, g in zip(names, grads)})
    return out
