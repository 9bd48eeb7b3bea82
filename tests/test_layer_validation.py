"""Host-side checks of the layer operators and of gradient clipping, in the binding and at the C ABI, before any CUDA
call (no GPU needed)."""
import ctypes
import types

import pytest
import torch

from paper_2609_13846_gb300 import dtp

vp = ctypes.c_void_p
OK, BAD = vp(1 << 20), vp((1 << 20) + 2)
BIG = 1 << 62


@pytest.fixture(scope="module")
def lib():
    from paper_2609_13846_gb300 import build
    build.build()
    return dtp.lib()


def _bf16(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def test_binding_rejects_host_tensors_and_names_them():
    with pytest.raises(ValueError, match="X must be a contiguous CUDA"):
        dtp.linear(_bf16(4, 8), _bf16(16, 8))
    with pytest.raises(ValueError, match="CUDA"):
        dtp.linear_backward(_bf16(4, 16), _bf16(4, 8), _bf16(16, 8))
    with pytest.raises(ValueError, match="CUDA"):
        dtp.gated_ffn(_bf16(4, 8), _bf16(16, 8), _bf16(16, 8), _bf16(8, 16))
    with pytest.raises(ValueError, match="CUDA"):
        dtp.gated_ffn_backward(_bf16(4, 8), _bf16(4, 8), _bf16(16, 8), _bf16(16, 8), _bf16(8, 16), (None, None))
    with pytest.raises(ValueError, match="CUDA"):
        dtp.clip_grad_norm([_bf16(4)], 1.0)
    with pytest.raises(ValueError, match="at least one"):
        dtp.clip_grad_norm([], 1.0)
    with pytest.raises(ValueError, match="shapes"):
        dtp.linear(_bf16(8), _bf16(16, 8))


@pytest.mark.parametrize("args", [(-1, 8, 8, 0, 0), (4, 0, 8, 0, 0), (4, 8, 0, 0, 0), (4, 8, 8, 2, 0), (4, 1 << 25, 8, 0, 1),
                                  ((1 << 31) - 255, 8, 8, 0, 0)])
def test_size_queries_reject_bad_sizes(lib, args):
    n = ctypes.c_size_t(0)
    assert lib.dtp_linear_workspace_size(*args, ctypes.byref(n)) == dtp.DTP_ERR_ARG
    assert lib.dtp_gated_ffn_workspace_size(*args, ctypes.byref(n)) == dtp.DTP_ERR_ARG


def test_workspace_sizes(lib):
    # aligned rows need no copies: the status header alone; odd ones a copy of X and of W at a pitch of 8 elements
    for T, K, N, want in ((100, 64, 32, 0), (100, 65, 32, (100 + 32) * 72 * 2)):
        n = dtp._size_query("dtp_linear_workspace_size", T, K, N, dtp.DTP_BF16, 0)
        assert want + 256 <= n <= want + 256 + 3 * 256
    assert dtp._size_query("dtp_linear_workspace_size", 100, 65, 32, dtp.DTP_F32, 0) <= 512
    both = dtp._size_query("dtp_gated_ffn_workspace_size", 100, 64, 96, dtp.DTP_BF16, 1)
    assert both >= dtp._size_query("dtp_gated_ffn_workspace_size", 100, 64, 96, dtp.DTP_BF16, 0) + 100 * 96 * 2
    assert dtp._size_query("dtp_gated_ffn_saved_size", 129, 130) == 2 * 2 * 2 * 128 * 128 * 4
    assert dtp._size_query("dtp_gated_ffn_saved_size", 0, 130) == 0


def test_linear_rejects_before_launch(lib):
    ok = [OK, OK, None, None, 4, 8, 8, 0, 0, OK, None, OK, BIG, None]
    for at, value, want in ((0, None, -1), (0, BAD, -1), (1, None, -1), (2, BAD, -1), (3, BAD, -1), (9, None, -1), (10, BAD, -1),
                            (7, 4, -1), (7, -1, -1), (8, 5, -1), (5, 0, -1), (11, None, -5), (12, 16, -5)):
        args = list(ok)
        args[at] = value
        assert lib.dtp_linear(*args) == want, (at, value)
    args = [None, None, None, None, 0, 8, 8, 0, 0, None, None, None, 0, None]
    assert lib.dtp_linear(*args) == dtp.DTP_OK                 # no tokens: nothing to do


def test_linear_backward_rejects_before_launch(lib):
    #     dY  X   W   Z     T  K  N act dtype dX  dW  db    ws  bytes stream
    ok = [OK, OK, OK, OK, 4, 8, 8, 1, 0, OK, OK, None, OK, BIG, None]
    for at, value, want in ((0, None, -1), (1, None, -1), (2, None, -1), (3, None, -1), (9, BAD, -1), (10, BAD, -1),
                            (11, BAD, -1), (7, 9, -1), (12, None, -5), (13, 300, -5)):
        args = list(ok)
        args[at] = value
        assert lib.dtp_linear_backward(*args) == want, (at, value)


def test_gated_rejects_before_launch(lib):
    ok = [OK, OK, OK, OK, None, 4, 8, 8, 1, 0, OK, None, None, OK, BIG, None]
    for at, value, want in ((0, None, -1), (1, BAD, -1), (2, None, -1), (3, None, -1), (4, BAD, -1), (10, None, -1), (11, BAD, -1),
                            (12, BAD, -1), (8, 7, -1), (13, None, -5), (14, 260, -5)):
        args = list(ok)
        args[at] = value
        assert lib.dtp_gated_ffn(*args) == want, (at, value)
    ok = [OK, OK, OK, OK, OK, OK, OK, 4, 8, 8, 1, 0, OK, OK, OK, OK, OK, BIG, None]
    for at, value, want in ((0, None, -1), (5, None, -1), (6, None, -1), (6, BAD, -1), (12, BAD, -1), (15, BAD, -1), (16, None, -5),
                            (17, 300, -5)):
        args = list(ok)
        args[at] = value
        assert lib.dtp_gated_ffn_backward(*args) == want, (at, value)


def test_clip_rejects_before_launch(lib):
    def call(ptrs=(1 << 20,), out=None, numel=(10,), dtypes=(1,), count=None, max_norm=1.0, norm=OK, ws=OK, size=BIG):
        n = len(numel)
        return lib.dtp_clip_grad_norm((vp * n)(*ptrs), None if out is None else (vp * n)(*out), (ctypes.c_int64 * n)(*numel),
                                      (ctypes.c_int * n)(*dtypes), n if count is None else count, max_norm, norm, ws, size, None)
    assert call(ptrs=(None,)) == -1
    assert call(ptrs=((1 << 20) + 2,)) == -1                    # fp32 on an odd half word
    assert call(ptrs=((1 << 20) + 1,), dtypes=(0,)) == -1
    assert call(out=(None,)) == -1
    assert call(numel=(-1,)) == -1 and call(numel=(1 << 47,)) == -1
    assert call(dtypes=(2,)) == -1 and call(count=-1) == -1
    assert call(max_norm=-1.0) == -1 and call(max_norm=float("nan")) == -1
    assert call(norm=None) == -1
    assert call(ws=None) == -5 and call(size=100) == -5
    n = ctypes.c_size_t(0)
    assert lib.dtp_clip_grad_norm_workspace_size(1, None, ctypes.byref(n)) == -1
    assert lib.dtp_clip_grad_norm_workspace_size(3000, (ctypes.c_int64 * 3000)(*[7] * 3000), ctypes.byref(n)) == 0
    assert n.value >= 256


@pytest.mark.parametrize("fn", ["dtp_linear_workspace_size", "dtp_gated_ffn_workspace_size"])
def test_widths_whose_sums_one_accumulator_holds(lib, fn):
    """2^20 terms lose about 2^-10 of their sum in one accumulator; wider sums are refused."""
    n = ctypes.c_size_t(0)
    for K, N, want in ((1 << 20, 8, 0), (8, 1 << 20, 0), ((1 << 20) + 1, 8, -1), (8, (1 << 20) + 1, -1)):
        assert getattr(lib, fn)(4, K, N, dtp.DTP_BF16, 1, ctypes.byref(n)) == want
    assert lib.dtp_gated_ffn_saved_size(4, (1 << 20) + 1, ctypes.byref(n)) == -1


def test_workspace_of_long_sums(lib):
    """A slot of fp32 sums for every 2^18 tokens of a weight gradient, none below."""
    def bytes_of(fn, T, K, N):
        return dtp._size_query(fn, T, K, N, dtp.DTP_F32, 1)

    T, K, N = 3 << 18, 24, 40
    for fn, per_token in (("dtp_linear_workspace_size", 4 * N + N / 8), ("dtp_gated_ffn_workspace_size", 8 * N)):
        more = bytes_of(fn, T, K, N) - T * per_token
        assert 3 * K * N * 4 <= more <= 3 * K * N * 4 + 5 * 256
        assert bytes_of(fn, 1 << 18, K, N) - (1 << 18) * per_token <= 5 * 256


def test_tensors_and_streams_of_another_device(monkeypatch):
    """The library launches on the current device: tensors or a stream of another one are refused."""
    monkeypatch.setattr(dtp, "_current_device", lambda: 0)
    with pytest.raises(ValueError, match="current device is cuda:0"):
        dtp._layer_stream(None, 1)
    with pytest.raises(ValueError, match="current device is cuda:0"):
        dtp._layer_stream(types.SimpleNamespace(device_index=1, cuda_stream=16), 1)
    with pytest.raises(ValueError, match="stream must be on cuda:0"):
        dtp._layer_stream(types.SimpleNamespace(device_index=1, cuda_stream=16), 0)
    assert dtp._layer_stream(types.SimpleNamespace(device_index=0, cuda_stream=16), 0) == 16


def test_workspaces_that_are_none():
    """Anything but bytes on the inputs' device: its pointer and its number of elements go to the library as they are."""
    for t in (torch.empty(4096, dtype=torch.uint8), torch.empty(4096, dtype=torch.uint8, device="meta")):
        with pytest.raises(ValueError, match="workspace must be"):
            dtp._workspace_check(t, 0)


def test_widths_that_are_no_c_int(lib):
    """2^32 + 8 columns are not 8."""
    wide = (1 << 32) + 8
    for fn in (dtp.linear_workspace, dtp.gated_ffn_workspace):
        for K, N in ((wide, 8), (8, wide), (1 << 31, 8)):
            with pytest.raises(ValueError, match="below 2\\^31"):
                fn(4, K, N, torch.bfloat16, "cpu")

    def meta(*shape):
        return torch.empty(shape, dtype=torch.bfloat16, device="meta")

    for K, N in ((wide, 8), (8, wide)):
        with pytest.raises(ValueError, match="below 2\\^31"):
            dtp.linear(meta(4, K), meta(N, K))
        with pytest.raises(ValueError, match="below 2\\^31"):
            dtp.gated_ffn(meta(4, K), meta(N, K), meta(N, K), meta(K, N))
