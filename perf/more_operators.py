"""The measured cases of a training step's other operators: the RMS norm, softmax cross entropy over a large vocabulary
from the hidden states, and the AdamW step over many tensors.

A permuted model that is distilled or evaluated runs a norm before each product, a loss over its vocabulary behind the last
one, and an update of all its weights.  Each listed case is one such call (a training case of the norm or the loss: forward
and backward) at widths of the repository's workloads, or generic odd ones; ``draw`` spreads the same calls over the whole
range of sizes.

A case is a dict with the operator ``op`` ("norm", "loss" or "adamw") and its sizes:
  norm:  T tokens, d width, residual (a gradient that joins the input's), train, dtype
  loss:  T tokens, d width, V vocabulary, ignored (share of the tokens without a target), train, dtype
  adamw: tensors, total (elements, about), tight (packed without alignment), shape_seed; layers > 0 gives the tensors of so many
         layers of the 1536-wide workload instead, and total = 0 its vectors alone; params and grads ("f32" or "bf16"), bits of
         the states, copies (bf16 ones of fp32 parameters), ratio (gradient norm over the limit; 0: no norm given)
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6
IGNORE = -100


def listed():
    return [
        # serving: the norm of one token of the 4096-wide workload
        dict(name="norm_token", op="norm", dtype="bf16", T=1, d=4096, residual=False, train=False),
        # training: a token batch through a norm of the 4096-wide workload, the residual stream's gradient added
        dict(name="norm_train", op="norm", dtype="bf16", T=16384, d=4096, residual=True, train=True),
        # the tight-check mode at odd sizes
        dict(name="norm_train_f32_odd", op="norm", dtype="f32", T=1003, d=1537, residual=False, train=True),
        # evaluation: the likelihood of one token, a large vocabulary
        dict(name="loss_token", op="loss", dtype="bf16", T=1, d=1024, V=131072, ignored=0.0, train=False),
        # evaluation: a text of odd length, an odd vocabulary
        dict(name="loss_text", op="loss", dtype="bf16", T=1003, d=1536, V=99991, ignored=0.0, train=False),
        # a training step's loss and gradients, a large vocabulary behind a narrow model; a tenth of the tokens is padding
        dict(name="loss_train", op="loss", dtype="bf16", T=8192, d=1024, V=131072, ignored=0.1, train=True),
        # the same behind the widest model
        dict(name="loss_train_wide", op="loss", dtype="bf16", T=4096, d=4096, V=65536, ignored=0.1, train=True),
        # the tight-check mode at odd sizes
        dict(name="loss_train_f32_odd", op="loss", dtype="f32", T=257, d=520, V=5003, ignored=0.3, train=True),
        # the smallest update: the vectors of one layer
        dict(name="adamw_vectors", op="adamw", layers=1, tensors=0, total=0, tight=False, shape_seed=0, params="f32",
             grads="f32", bits=32, copies=False, ratio=0.0),
        # mixed-precision training of a 16-layer model: fp32 master weights, bf16 gradients over the limit, bf16 copies
        dict(name="adamw_model", op="adamw", layers=16, tensors=0, total=1, tight=False, shape_seed=0, params="f32",
             grads="bf16", bits=32, copies=True, ratio=3.7),
        # the same with states in 8 bits
        dict(name="adamw_model_8bit", op="adamw", layers=16, tensors=0, total=1, tight=False, shape_seed=0, params="f32",
             grads="bf16", bits=8, copies=True, ratio=3.7),
        # bf16 weights without a master copy, many odd tensors packed without alignment, states in 8 bits
        dict(name="adamw_tight_8bit", op="adamw", layers=0, tensors=301, total=60_000_000, tight=True, shape_seed=7,
             params="bf16", grads="bf16", bits=8, copies=False, ratio=0.5),
    ]


# ------------------------------------------------------------------------ draws --

MOST_FLOPS = 6.5e12
MOST_VALUES = 16384 * 4096
MOST_ELEMENTS = 380_000_000


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A layer's width: a common one, any multiple of 8, or any number."""
    kind = rng.random()
    if kind < 0.4:
        return rng.choice([w for w in (64, 768, 1024, 1536, 2048, 4096, 8192) if lo <= w <= hi])
    w = _log(rng, lo, hi)
    return max(8, w // 8 * 8) if kind < 0.8 else w


def draw(rng):
    op = rng.choice(["norm", "norm", "loss", "loss", "loss", "adamw", "adamw", "adamw"])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    train = rng.random() < 0.6
    if op == "norm":
        c = dict(op=op, dtype=dtype, T=_log(rng, 1, 65536), d=_width(rng, 64, 8192), residual=rng.random() < 0.5, train=train)
        while c["T"] * c["d"] * _e(c) > 2 * MOST_VALUES:
            c["T"] = c["T"] * 2 // 3
        return c
    if op == "loss":
        V = rng.choice([32768, 65536, 131072]) if rng.random() < 0.4 else _log(rng, 100, 131072)
        c = dict(op=op, dtype=dtype, T=_log(rng, 1, 16384), d=_width(rng, 64, 4096), V=V,
                 ignored=rng.choice([0.0, 0.1, 0.5]), train=train)
        while work(c)["flops"] > (MOST_FLOPS if dtype == "bf16" else MOST_FLOPS / 8) or c["T"] * V > 8192 * 131072:
            c["T"] = c["T"] * 2 // 3
        return c
    total = _log(rng, 2000, MOST_ELEMENTS)
    params = rng.choice(["f32", "f32", "bf16"])
    return dict(op=op, layers=0, tensors=min(_log(rng, 1, 400), total), total=total, tight=rng.random() < 0.4,
                shape_seed=rng.randrange(1 << 20), params=params, grads=rng.choice(["f32", "bf16", "bf16"]),
                bits=rng.choice([8, 32]), copies=params == "f32" and rng.random() < 0.6, ratio=rng.choice([0.0, 0.5, 3.7]))


# ------------------------------------------------------------------------- work --

def _e(c):
    return 2 if c["dtype"] == "bf16" else 4


def work(c):
    if c["op"] == "norm":
        n, e = c["T"] * c["d"], _e(c)
        values = 2 * n + (2 * n + n * c["residual"] if c["train"] else 0)      # x, y; dy, dx, the residual's gradient
        return dict(bytes=values * e + 4 * c["d"] * (2 if c["train"] else 1) + 4 * c["T"],
                    flops=(16 if c["train"] else 4) * n)
    if c["op"] == "loss":
        T, d, V = c["T"], c["d"], c["V"]
        values = (T + V) * d * (2 if c["train"] else 1)
        return dict(bytes=values * _e(c) + T * 16, flops=(6 if c["train"] else 2) * T * d * V)
    n = sum(_sizes(c))
    p, g, s = (4 if c["params"] == "f32" else 2), (4 if c["grads"] == "f32" else 2), c["bits"] // 8
    scales = 16 * sum((k + BLOCK - 1) // BLOCK for k in _sizes(c)) if c["bits"] == 8 else 0
    return dict(bytes=n * (2 * p + g + 4 * s + 2 * c["copies"]) + scales, flops=16 * n)


# ----------------------------------------------------------------------- inputs --

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, std, dtype):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).mul_(std).to(dtype)


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _sizes(c):
    """Elements of each of the case's tensors."""
    if c["layers"]:
        d, N, q, kv = 1536, 4096, 1536, 768
        vectors = [d, d, 96, 96]
        layer = [q * d, kv * d, kv * d, d * q, N * d, N * d, d * N] + vectors
        return (layer if c["total"] else vectors) * c["layers"]
    r = random.Random(c["shape_seed"])
    w = [math.exp(r.gauss(0.0, 2.0)) for _ in range(c["tensors"])]
    s = sum(w)
    return [max(1, int(c["total"] * x / s)) for x in w]


def prepare(c, seed):
    g = _gen(seed)
    if c["op"] == "adamw":
        return _prepare_adamw(c, g)
    dt, T, d = _dtype(c["dtype"]), c["T"], c["d"]
    # hidden states: N(0,1) with 4 outlier channels scaled by 20, as in the calibration workloads
    x = torch.randn((T, d), generator=g, device=DEV, dtype=torch.float32)
    outliers = torch.randperm(d, generator=g, device=DEV)[:4]
    s = dict(case=c)
    if c["op"] == "norm":
        x[:, outliers] *= 20.0
        s.update(X=x.to(dt), gamma=1.0 + _normal(g, (d,), 0.2, torch.float32))
        if c["train"]:
            s.update(dY=_normal(g, (T, d), 1e-2, dt), dres=_normal(g, (T, d), 1e-2, dt) if c["residual"] else None)
        if own and c["train"]:         # the workspace that a training loop keeps
            from paper_2609_13846_gb300 import dtp
            s["workspace"] = dtp.rms_norm_workspace(T, d, dt, DEV)
        return s
    x[:, outliers] *= 4.0
    # logits of a few units, as a trained model's
    s.update(X=x.to(dt), W=_normal(g, (c["V"], d), 2.0 / math.sqrt(d), dt))
    targets = torch.randint(0, c["V"], (T,), generator=g, device=DEV)
    padding = torch.rand((T,), generator=g, device=DEV) < c["ignored"]
    s["targets"] = torch.where(padding, torch.full_like(targets, IGNORE), targets)
    if c["train"]:                     # the gradient of a mean over the tokens with a target
        count = (s["targets"] != IGNORE).sum().clamp(min=1)
        s["dloss"] = (torch.ones(T, device=DEV) / count).float()
    if own:
        from paper_2609_13846_gb300 import dtp
        s["workspace"] = dtp.linear_cross_entropy_workspace(T, d, c["V"], dt, DEV, backward=c["train"])
    return s


BLOCK = 256        # elements that share a scale in the 8-bit states


def _flat(sizes, tight, dtype, per=1):
    """(one buffer, a view of it for each size); ``per`` elements to a value."""
    counts = [-(-n // per) for n in sizes]
    starts, used = [], 0
    for n in counts:
        starts.append(used)
        used += n if tight else (n + 63) // 64 * 64
    buffer = torch.zeros(used, device=DEV, dtype=dtype)
    return buffer, [buffer[at:at + n] for at, n in zip(starts, counts)]


def _prepare_adamw(c, g):
    sizes, tight, eight = _sizes(c), c["tight"], c["bits"] == 8
    s = dict(case=c, lr=1e-4, betas=(0.9, 0.999), eps=1e-8, decay=0.1, norm=None, limit=math.inf, copies=None)
    s["params"], params = _flat(sizes, tight, _dtype(c["params"]))
    grads_flat, grads = _flat(sizes, tight, _dtype(c["grads"]))
    held = torch.float8_e4m3fn if eight else torch.float32
    s["m"], m = _flat(sizes, tight, held)
    s["v"], v = _flat(sizes, tight, held)
    state = dict(bits=c["bits"], m=m, v=v, m_scale=None, v_scale=None,
                 step=torch.full((), 100, dtype=torch.int64, device=DEV))
    if eight:
        s["m_scale"], state["m_scale"] = _flat(sizes, False, torch.float32, BLOCK)
        s["v_scale"], state["v_scale"] = _flat(sizes, False, torch.float32, BLOCK)
    for i, n in enumerate(sizes):
        std = 10.0 ** -(1 + i % 4)     # gradients of layers differ in scale by orders of magnitude
        params[i].copy_(_normal(g, (n,), 0.02, torch.float32))
        grads[i].copy_(_normal(g, (n,), std, torch.float32))
        first = _normal(g, (n,), 0.3 * std, torch.float32)
        root = torch.rand((n,), generator=g, device=DEV).add_(0.5).mul_(std)
        if eight:
            u = torch.full((n,), 0.5, device=DEV)
            code, state["m_scale"][i][:] = _encode(first, u)
            m[i].view(torch.uint8).copy_(code)
            code, state["v_scale"][i][:] = _encode(root, u)
            v[i].view(torch.uint8).copy_(code)
        else:
            m[i].copy_(first)
            v[i].copy_(root.square())
    s.update(param_list=params, grads=grads, state=state)
    if c["copies"]:
        s["copy"], s["copies"] = _flat(sizes, tight, torch.bfloat16)
    if c["ratio"] > 0:
        s["norm"] = grads_flat.double().square().sum().sqrt().float()
        s["limit"] = float(s["norm"]) / c["ratio"]
    if own:
        from paper_2609_13846_gb300 import dtp
        s["workspace"] = dtp.adamw_workspace(params)
    return s


# ------------------------------------------------------------------ plain forms --

def _plain_norm(s):
    c, x, gamma = s["case"], s["X"].float(), s["gamma"]
    rms = (x.square().mean(-1) + EPS).sqrt()
    n = x / rms[:, None]
    out = dict(Y=(n * gamma).to(s["X"].dtype), rms=rms)
    if c["train"]:
        dy = s["dY"].float()
        dn = dy * gamma
        dx = (dn - n * (dn * n).mean(-1, keepdim=True)) / rms[:, None]
        if s["dres"] is not None:
            dx = dx + s["dres"].float()
        out.update(dX=dx.to(s["X"].dtype), dgamma=(dy * n).sum(0))
    return out


def _plain_loss(s):
    x, w, y = s["X"].float(), s["W"].float(), s["targets"]
    z = x @ w.t()
    top = z.max(1).values
    lse = top + torch.log(torch.exp(z - top[:, None]).sum(1))
    some = y != IGNORE
    at = torch.where(some, y, torch.zeros_like(y))[:, None]
    out = dict(loss=torch.where(some, lse - z.gather(1, at)[:, 0], torch.zeros_like(lse)), lse=lse)
    if s["case"]["train"]:
        g = torch.where(some, s["dloss"], torch.zeros_like(lse))[:, None]
        dz = torch.exp(z - lse[:, None]) * g
        dz.scatter_add_(1, at, -g)
        out.update(dX=(dz @ w).to(s["X"].dtype), dW=(dz.t() @ x).to(s["W"].dtype))
    return out


def _uniform(n, step):
    """Three numbers in [0, 2^32) for each of n elements: mixes of its index and the step in 32-bit arithmetic (two rounds of
    xor-shift and multiply, then a multiply for each of the other two)."""
    mask = 0xFFFFFFFF
    i = torch.arange(n, device=DEV)
    x = (i + (i >> 32) * 0x85EBCA6B + step * 0x9E3779B9) & mask
    x = ((x ^ (x >> 16)) * 0x7FEB352D) & mask
    x = ((x ^ (x >> 15)) * 0x846CA68B) & mask
    x = x ^ (x >> 16)
    return x, (x * 0x9E3779B1) & mask, (x * 0x85EBCA77) & mask


def _fraction(x):
    """[0, 2^32) to [0, 1) in 23 bits."""
    return (x >> 9).float() * 2.0 ** -23


def _blocks(x):
    return torch.nn.functional.pad(x, (0, -x.numel() % BLOCK)).view(-1, BLOCK)


def _encode(x, u):
    """(e4m3 codes of x over its block's scale, rounded up where the fraction of the step and ``u`` reach 1, scales): the
    largest finite size of a block stands for 448; what is not finite is held as NaN."""
    b = _blocks(x)
    fine = torch.isfinite(b)
    top = torch.where(fine, b.abs(), torch.zeros_like(b)).max(1).values
    live = top >= 2.0 ** -100
    up = torch.where(live, 448.0 / top, torch.zeros_like(top))
    a = (b.abs() * up[:, None]).view(-1)[:x.numel()]
    exponent = (a.view(torch.int32) & 0x7F800000).clamp(min=121 << 23)           # of at least 2^-6
    per_step = ((128 << 23) - exponent + (129 << 23)).view(torch.float32)          # 8 steps to a binade
    code = ((exponent - (121 << 23)) >> 20) + torch.floor(a * per_step + u).nan_to_num(0.0, 0.0, 0.0).int()
    code = code.clamp(max=0x7E) + 128 * (x < 0).int()
    return torch.where(torch.isfinite(x), code, 0x7F).to(torch.uint8), torch.where(live, top / 448.0, torch.zeros_like(top))


def _decode(code, scale):
    return (_blocks(code.float()) * scale[:, None]).view(-1)[:code.numel()]


def _plain_adamw_tensor(s, i, f):
    """One tensor's update with the step's factors f, in place."""
    p, st, eight = s["param_list"][i], s["state"], s["case"]["bits"] == 8
    g = s["grads"][i].float() * f["clip"]
    m = _decode(st["m"][i], st["m_scale"][i]) if eight else st["m"][i]
    v = _decode(st["v"][i], st["v_scale"][i]).square() if eight else st["v"][i]
    m = m * f["b1"] + g * f["1-b1"]
    v = v * f["b2"] + g * g * f["1-b2"]
    root = v.sqrt()
    new = p.float() * f["keep"] - f["size"] * (m / (root * f["root"] + s["eps"]))
    low = p.dtype == torch.bfloat16
    r = _uniform(p.numel(), f["step"]) if eight or low else None
    if low:          # no master copy: up or down in proportion, so that small updates are not lost
        bits = (new.view(torch.int32) + (r[2] >> 16).int()) & -65536
        new = torch.where(torch.isfinite(new), bits.view(torch.float32), new)
    p.copy_(new)
    if eight:
        code, scale = _encode(m, _fraction(r[0]))
        st["m"][i].view(torch.uint8).copy_(code)
        st["m_scale"][i].copy_(scale)
        code, scale = _encode(root, _fraction(r[1]))
        code = torch.where((root > 0) & (code == 0), torch.ones_like(code), code)      # a moment is never lost
        st["v"][i].view(torch.uint8).copy_(code)
        st["v_scale"][i].copy_(scale)
    else:
        st["m"][i].copy_(m)
        st["v"][i].copy_(v)
    if s["copies"] is not None:
        s["copies"][i].copy_(new)


def _plain_adamw(s):
    (b1, b2), lr, state = s["betas"], s["lr"], s["state"]
    state["step"] += 1
    t = state["step"].double()
    clip = torch.ones((), device=DEV) if s["norm"] is None else torch.clamp(s["limit"] / s["norm"], max=1.0)
    f = {"b1": b1, "1-b1": 1.0 - b1, "b2": b2, "1-b2": 1.0 - b2, "keep": 1.0 - lr * s["decay"], "clip": clip,
         "size": (lr / -torch.expm1(t * math.log(b1))).float(), "root": (-torch.expm1(t * math.log(b2))).rsqrt().float(),
         "step": state["step"]}
    [_plain_adamw_tensor(s, i, f) for i in range(len(s["param_list"]))]
    return _adamw_outputs(s)


def _adamw_outputs(s):
    """The updated buffers; 8-bit states as the e4m3 values that they hold, with their scales."""
    names = ["params", "m", "v"] + ["m_scale", "v_scale"] * (s["case"]["bits"] == 8) + ["copy"] * s["case"]["copies"]
    return {k: s[k] for k in names}


# ------------------------------------------------------------------- the passes --

def run(s):
    c = s["case"]
    if not own:
        return dict(norm=_plain_norm, loss=_plain_loss, adamw=_plain_adamw)[c["op"]](s)
    from paper_2609_13846_gb300 import dtp
    if c["op"] == "norm":
        y, rms = dtp.rms_norm(s["X"], s["gamma"], eps=EPS)
        out = dict(Y=y, rms=rms)
        if c["train"]:
            out["dX"], out["dgamma"] = dtp.rms_norm_backward(s["dY"], s["X"], s["gamma"], rms, dresidual=s["dres"],
                                                             workspace=s["workspace"])
        return out
    if c["op"] == "loss":
        loss, lse = dtp.linear_cross_entropy(s["X"], s["W"], s["targets"], ignore_index=IGNORE, workspace=s["workspace"])
        out = dict(loss=loss, lse=lse)
        if c["train"]:
            out["dX"], out["dW"] = dtp.linear_cross_entropy_backward(s["dloss"], s["X"], s["W"], s["targets"], lse,
                                                                     ignore_index=IGNORE, workspace=s["workspace"])
        return out
    dtp.adamw_step(s["param_list"], s["grads"], s["state"], lr=s["lr"], betas=s["betas"], eps=s["eps"],
                   weight_decay=s["decay"], norm=s["norm"], max_norm=s["limit"], copies=s["copies"],
                   workspace=s["workspace"])
    return _adamw_outputs(s)


# ---------------------------------------------------------------- exact results --

EXACT_FLOPS = 7e12      # about 12 s of fp64 on the GPU


def _exact_norm(s):
    x = s["X"].to(torch.float64).requires_grad_()
    gamma = s["gamma"].to(torch.float64).requires_grad_()
    rms = torch.sqrt(torch.einsum("td,td->t", x, x) / x.shape[1] + EPS)
    y = torch.einsum("td,t,d->td", x, 1.0 / rms, gamma)
    out = dict(Y=y.detach(), rms=rms.detach())
    if s["case"]["train"]:
        dx, out["dgamma"] = torch.autograd.grad(y, (x, gamma), s["dY"].to(torch.float64))
        out["dX"] = dx if s["dres"] is None else dx + s["dres"].to(torch.float64)
    return out


def _exact_loss(s):
    """Token by token in slices, so that the logits in 64 bits fit; the gradients from softmax written out."""
    T, V = s["X"].shape[0], s["W"].shape[0]
    w = s["W"].to(torch.float64)
    train = s["case"]["train"]
    loss, lses, dx, dw = [], [], [], torch.zeros_like(w) if train else None
    for t0 in range(0, T, 2048):
        x, y = s["X"][t0:t0 + 2048].to(torch.float64), s["targets"][t0:t0 + 2048]
        z = torch.einsum("td,vd->tv", x, w)
        lse = torch.logsumexp(z, 1)
        hit = torch.arange(V, device=DEV)[None, :] == y[:, None]
        lses.append(lse)
        loss.append(torch.where(y == IGNORE, 0.0, lse - torch.where(hit, z, 0.0).sum(1)))
        if train:
            g = torch.where(y == IGNORE, 0.0, s["dloss"][t0:t0 + 2048].to(torch.float64))
            z = torch.softmax(z, 1).sub_(hit.to(torch.float64)).mul_(g[:, None])
            dx.append(torch.einsum("tv,vd->td", z, w))
            dw += torch.einsum("tv,td->vd", z, x)
    out = dict(loss=torch.cat(loss), lse=torch.cat(lses))
    if train:
        out.update(dX=torch.cat(dx), dW=dw)
    return out


def _exact_adamw(s):
    """The update written out in 64 bits; the states that are held in 8 bits before their rounding, over the exact scale."""
    c, st, d = s["case"], s["state"], torch.float64
    eight = c["bits"] == 8
    (b1, b2), t = s["betas"], int(st["step"]) + 1
    factor = 1.0 if s["norm"] is None else min(1.0, s["limit"] / float(s["norm"]))
    out = {k: torch.zeros(s[k].shape, dtype=d, device=DEV) for k in _adamw_outputs(s)}

    def place(k, like, value):
        at = like.storage_offset()
        out[k][at:at + value.numel()] = value

    for i, p in enumerate(s["param_list"]):
        n = p.numel()

        def held(k):
            x = st[k][i].to(torch.float32).to(d)
            return x * st[k + "_scale"][i].to(d).repeat_interleave(BLOCK)[:n] if eight else x

        g = s["grads"][i].to(d) * factor
        m = held("m") + (1.0 - b1) * (g - held("m"))
        old = held("v") ** 2 if eight else held("v")
        v = old + (1.0 - b2) * (g * g - old)
        q = p.to(d)
        q = q - s["lr"] * s["decay"] * q - s["lr"] * (m / (1.0 - b1 ** t)) / (torch.sqrt(v / (1.0 - b2 ** t)) + s["eps"])
        place("params", p, q)
        if c["copies"]:
            place("copy", s["copies"][i], q)
        if not eight:
            place("m", st["m"][i], m)
            place("v", st["v"][i], v)
            continue
        for k, x in (("m", m), ("v", torch.sqrt(v))):
            scale = torch.nn.functional.pad(x.abs(), (0, -n % BLOCK)).view(-1, BLOCK).amax(1) / 448.0
            place(k + "_scale", st[k + "_scale"][i], scale)
            place(k, st[k][i], x / scale.repeat_interleave(BLOCK)[:n])
    return out


def exact(c, seed):
    if c["op"] == "loss" and work(c)["flops"] > EXACT_FLOPS:
        return None
    return dict(norm=_exact_norm, loss=_exact_loss, adamw=_exact_adamw)[c["op"]](prepare(c, seed))
