"""Host-side checks of the norm, the vocabulary's loss and the update, in the binding and at the C ABI, before any CUDA call
(no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2609_13846_gb300 import dtp

vp = ctypes.c_void_p
OK, ODD, BAD = vp(1 << 20), vp((1 << 20) + 4), vp((1 << 20) + 1)
BIG = 1 << 62


@pytest.fixture(scope="module")
def lib():
    from paper_2609_13846_gb300 import build
    build.build()
    return dtp.lib()


def _refuses(fn, ok, cases):
    for at, value, want in cases:
        args = list(ok)
        args[at] = value
        assert fn(*args) == want, (at, value)


def test_binding_names_what_is_wrong():
    x, w, gamma = (torch.zeros(s, dtype=t) for s, t in (((4, 8), torch.bfloat16), ((16, 8), torch.bfloat16), ((8,), torch.float32)))
    y, f = torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    with pytest.raises(ValueError, match="X must be a contiguous CUDA"):
        dtp.rms_norm(x, gamma)
    with pytest.raises(ValueError, match="X must be"):
        dtp.rms_norm(x[0], gamma)
    with pytest.raises(ValueError, match="CUDA"):
        dtp.rms_norm_backward(x, x, gamma, f)
    with pytest.raises(ValueError, match="CUDA"):
        dtp.linear_cross_entropy(x, w, y)
    with pytest.raises(ValueError, match="CUDA"):
        dtp.linear_cross_entropy_backward(f, x, w, y, f)
    with pytest.raises(ValueError, match="params must be contiguous CUDA"):
        dtp.adamw_step([gamma], [gamma], dtp.adamw_state([gamma]), lr=1e-3)
    with pytest.raises(ValueError, match="at least one"):
        dtp.adamw_step([], [], {}, lr=1e-3)
    for call in (dtp.adamw_state, dtp.adamw_workspace):
        with pytest.raises(ValueError, match="at least one"):
            call([])
    with pytest.raises(ValueError, match="bits"):
        dtp.adamw_state([gamma], bits=16)


def test_states():
    p = [torch.zeros(3, 100), torch.zeros(0), torch.zeros(256)]
    s = dtp.adamw_state(p)
    assert [t.shape[0] for t in s["m"]] == [300, 0, 256] and s["m"][0].dtype is torch.float32 and s["m_scale"] is None
    s = dtp.adamw_state(p, bits=8)
    assert [t.shape[0] for t in s["v_scale"]] == [2, 0, 1] and s["v"][0].dtype is torch.float8_e4m3fn
    assert s["step"].dtype is torch.int64 and s["step"].shape == ()
    m, v = dtp.adamw_moments(s)
    assert [t.shape[0] for t in m] == [300, 0, 256] and all((t == 0).all() for t in m + v)


@pytest.mark.parametrize("T,d", [(-1, 8), (4, 0), (4, 1 << 25), ((1 << 31) - 255, 8)])
def test_size_queries_reject_bad_sizes(lib, T, d):
    n = ctypes.c_size_t(0)
    assert lib.dtp_rms_norm_backward_workspace_size(T, d, ctypes.byref(n)) == dtp.DTP_ERR_ARG
    for args in ((T, d, 8), (T, 8, d)):
        if T == 4 or args[1] == d:
            assert lib.dtp_linear_cross_entropy_workspace_size(*args, 0, 0, ctypes.byref(n)) == dtp.DTP_ERR_ARG
    assert lib.dtp_linear_cross_entropy_workspace_size(4, 8, 8, 2, 0, ctypes.byref(n)) == dtp.DTP_ERR_ARG
    assert lib.dtp_adamw_workspace_size(-1, None, ctypes.byref(n)) == dtp.DTP_ERR_ARG
    bad = (ctypes.c_int64 * 1)(-5)
    assert lib.dtp_adamw_workspace_size(1, ctypes.cast(bad, vp), ctypes.byref(n)) == dtp.DTP_ERR_ARG


def test_workspaces_hold_a_piece_of_the_logits():
    """What a call takes does not grow with the vocabulary beyond a piece of it."""
    q = [dtp._size_query("dtp_linear_cross_entropy_workspace_size", 8192, 1024, V, dtp.DTP_BF16, 1) for V in (131072, 1048576)]
    assert q[1] - q[0] <= 8192 * (1048576 - 131072) // 16 and q[0] <= 3 << 30


def test_norm_rejects_before_launch(lib):
    ok = [OK, OK, 4, 8, 1e-6, 0, OK, OK, None]
    _refuses(lib.dtp_rms_norm, ok, [(0, None, -1), (0, BAD, -1), (1, None, -1), (1, vp((1 << 20) + 2), -1), (3, 0, -1), (4, 0.0, -1),
                                    (4, float("nan"), -1), (4, float("inf"), -1), (5, 3, -1), (6, None, -1), (7, BAD, -1), (2, -1, -1)])
    assert lib.dtp_rms_norm(None, None, 0, 8, 1e-6, 0, None, None, None) == dtp.DTP_OK
    ok = [OK, OK, OK, OK, None, 4, 8, 1, OK, OK, OK, BIG, None]
    _refuses(lib.dtp_rms_norm_backward, ok, [(0, None, -1), (0, vp((1 << 20) + 2), -1), (1, None, -1), (2, None, -1), (3, None, -1),
                                             (4, BAD, -1), (8, BAD, -1), (9, BAD, -1), (10, None, -5), (11, 16, -5), (7, 2, -1)])


def test_loss_rejects_before_launch(lib):
    #     X   W   targets T d V ignore dtype loss lse ws bytes stream
    ok = [OK, OK, OK, 4, 8, 16, -100, 0, OK, OK, OK, BIG, None]
    _refuses(lib.dtp_linear_cross_entropy, ok,
             [(0, None, -1), (0, ODD, -1), (1, None, -1), (1, ODD, -1), (2, None, -1), (2, ODD, -1), (8, None, -1), (8, BAD, -1),
              (9, None, -1), (10, None, -5), (11, 300, -5), (5, 0, -1), (7, 4, -1)])
    assert lib.dtp_linear_cross_entropy(None, None, None, 0, 8, 16, -100, 0, None, None, None, 0, None) == dtp.DTP_OK
    ok = [OK, OK, OK, OK, OK, 4, 8, 16, -100, 0, OK, OK, OK, BIG, None]
    _refuses(lib.dtp_linear_cross_entropy_backward, ok,
             [(0, None, -1), (0, BAD, -1), (1, None, -1), (2, ODD, -1), (3, ODD, -1), (4, None, -1), (10, ODD, -1), (11, ODD, -1),
              (12, None, -5), (13, 300, -5)])


def _opts(**more):
    o = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, max_norm=float("inf"), state_bits=32)
    o.update(more)
    return dtp.AdamWOpts(*o.values())


def _ptrs(*values):
    return ctypes.cast((vp * len(values))(*values), vp)


def _call(lib, opts, **more):
    one = _ptrs(1 << 20)
    codes = lambda c: ctypes.cast((ctypes.c_int * 1)(c), vp)  # noqa: E731
    a = dict(params=one, pd=codes(1), grads=one, gd=codes(0), m=one, v=one, ms=None, vs=None, copies=None,
             numel=ctypes.cast((ctypes.c_int64 * 1)(10), vp), count=1)
    rest = dict(lr=None, norm=None, step=OK, ws=OK, bytes=BIG, stream=None)
    for k, x in more.items():
        (a if k in a else rest)[k] = x
    return lib.dtp_adamw(*a.values(), ctypes.byref(opts) if opts else None, *rest.values())


def test_adamw_rejects_before_launch(lib):
    nan, inf = float("nan"), float("inf")
    for bad in (dict(lr=nan), dict(lr=inf), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=nan), dict(beta2=1.0), dict(eps=0.0),
                dict(eps=-1.0), dict(eps=1e-40), dict(weight_decay=inf), dict(max_norm=-1.0), dict(max_norm=nan), dict(state_bits=16)):
        assert _call(lib, _opts(**bad)) == dtp.DTP_ERR_ARG, bad
    held = _opts()
    held.reserved[2] = 1
    assert _call(lib, held) == _call(lib, None) == dtp.DTP_ERR_ARG
    code = lambda c: ctypes.cast((ctypes.c_int * 1)(c), vp)  # noqa: E731
    for bad in (dict(params=None), dict(params=_ptrs(None)), dict(params=_ptrs((1 << 20) + 2)), dict(grads=_ptrs((1 << 20) + 1)),
                dict(m=_ptrs((1 << 20) + 2)), dict(v=_ptrs(None)), dict(pd=code(2)), dict(gd=code(-1)), dict(step=None), dict(step=ODD),
                dict(lr=BAD), dict(norm=BAD), dict(count=-1), dict(copies=_ptrs((1 << 20) + 1)),
                dict(copies=_ptrs(1 << 20), pd=code(0)), dict(numel=ctypes.cast((ctypes.c_int64 * 1)(-1), vp))):
        assert _call(lib, _opts(), **bad) == dtp.DTP_ERR_ARG, bad
    assert _call(lib, _opts(state_bits=8)) == dtp.DTP_ERR_ARG                        # no scales
    assert _call(lib, _opts(state_bits=8), ms=_ptrs(1 << 20), vs=_ptrs((1 << 20) + 2)) == dtp.DTP_ERR_ARG
    assert _call(lib, _opts(), ws=None) == _call(lib, _opts(), bytes=300) == dtp.DTP_ERR_WORKSPACE
