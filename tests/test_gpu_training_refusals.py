"""What the norm, the vocabulary's loss and the update refuse, on GPU tensors, before anything is launched."""
import pytest
import torch

from paper_2609_13846_gb300 import dtp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _t(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype, device=DEV)


def test_norm_and_loss_refusals():
    x, g = _t(4, 16, dtype=torch.bfloat16), _t(16)
    w, y, f = _t(8, 16, dtype=torch.bfloat16), _t(4, dtype=torch.int64), _t(4)
    for call, error, text in (
            (lambda: dtp.rms_norm(x, g.bfloat16()), TypeError, "gamma"), (lambda: dtp.rms_norm(x.half(), g), TypeError, "float16"),
            (lambda: dtp.rms_norm(x.t(), _t(4)), ValueError, "contiguous"), (lambda: dtp.rms_norm(x, _t(15)), ValueError, "gamma"),
            (lambda: dtp.rms_norm(x, g, eps=0.0), dtp.DTPError, "argument"),
            (lambda: dtp.rms_norm(x, g, Y=_t(4, 16)), TypeError, "Y"), (lambda: dtp.rms_norm(x.cpu(), g.cpu()), ValueError, "CUDA"),
            (lambda: dtp.rms_norm_backward(x, x, g, _t(5)), ValueError, "rms"),
            (lambda: dtp.rms_norm_backward(x, x, g, f, dresidual=_t(4, 16)), TypeError, "dresidual"),
            (lambda: dtp.rms_norm_backward(x, x, g, f, workspace=_t(64)), ValueError, "workspace"),
            (lambda: dtp.rms_norm_backward(x, x, g, f, workspace=_t(64, dtype=torch.uint8)), dtp.DTPError, "workspace"),
            (lambda: dtp.linear_cross_entropy(x, w, y.int()), TypeError, "targets"),
            (lambda: dtp.linear_cross_entropy(x, w, y[:3]), ValueError, "targets"),
            (lambda: dtp.linear_cross_entropy(x, w.float(), y), TypeError, "W"),
            (lambda: dtp.linear_cross_entropy(x, w, y, ignore_index=1 << 63), ValueError, "ignore_index"),
            (lambda: dtp.linear_cross_entropy(x, w[:, :8], y), ValueError, "W"),
            (lambda: dtp.linear_cross_entropy_backward(f.double(), x, w, y, f), TypeError, "dloss"),
            (lambda: dtp.linear_cross_entropy_backward(f, x, w, y, f[:2]), ValueError, "lse"),
            (lambda: dtp.linear_cross_entropy_backward(f, x, w, y, f, workspace=_t(300, dtype=torch.uint8)), dtp.DTPError, "workspace")):
        with pytest.raises(error, match=text):
            call()


def test_update_refusals():
    p = [_t(10), _t(300)]
    s32, s8 = dtp.adamw_state(p), dtp.adamw_state(p, bits=8)
    step = lambda params=p, grads=p, state=s32, **more: dtp.adamw_step(params, grads, state, **dict(dict(lr=1e-3), **more))  # noqa: E731
    for call, error, text in (
            (lambda: step(grads=[p[0]]), ValueError, "as many"), (lambda: step(grads=[p[1], p[0]]), ValueError, "grads"),
            (lambda: step(grads=[p[0], p[1].half()]), TypeError, "grads"), (lambda: step(params=[p[0], p[1].double()]), TypeError, "params"),
            (lambda: step(params=[p[0], _t(2, 300)[:, ::2]]), ValueError, "contiguous"),
            (lambda: step(params=[p[1], p[1]], grads=[p[1], p[1]]), ValueError, "twice"),
            (lambda: step(params=[p[0], 3.0]), TypeError, "tensors"), (lambda: step(grads=[p[0], p[1].cpu()]), ValueError, "CUDA"),
            (lambda: step(state=dict(s32, bits=16)), ValueError, "bits"), (lambda: step(state=dict(s32, m=s8["m"])), TypeError, "moments"),
            (lambda: step(state=dict(s32, v=s32["v"][:1])), ValueError, "as many"),
            (lambda: step(state=dict(s8, v_scale=s8["v_scale"][::-1])), ValueError, "v_scale"),
            (lambda: step(state=dict(s8, m_scale=[t.half() for t in s8["m_scale"]])), TypeError, "scales"),
            (lambda: step(state=dict(s32, step=_t())), ValueError, "step"), (lambda: step(lr=_t(2)), ValueError, "lr"),
            (lambda: step(norm=_t(dtype=torch.float64)), ValueError, "norm"),
            (lambda: step(copies=[_t(10, dtype=torch.bfloat16)]), ValueError, "as many"),
            (lambda: step(copies=[_t(10), None]), TypeError, "copies"),
            (lambda: step(copies=[None, _t(10, dtype=torch.bfloat16)]), ValueError, "copies"),
            (lambda: step(params=[q.bfloat16() for q in p], copies=[_t(10, dtype=torch.bfloat16), None]), TypeError, "copies"),
            (lambda: step(betas=(1.0, 0.9)), dtp.DTPError, "argument"), (lambda: step(eps=0.0), dtp.DTPError, "argument"),
            (lambda: step(max_norm=-1.0), dtp.DTPError, "argument"), (lambda: step(lr=float("nan")), dtp.DTPError, "argument"),
            (lambda: step(workspace=_t(64)), ValueError, "workspace"),
            (lambda: step(workspace=_t(256, dtype=torch.uint8)), dtp.DTPError, "workspace")):
        with pytest.raises(error, match=text):
            call()
    assert int(s32["step"]) == int(s8["step"]) == 0 and all((q == 0).all() for q in p)
    step(copies=[None, None])
    assert int(s32["step"]) == 1
