"""Rules of the sources of the norm, the vocabulary's loss and the update that a run on the GPU cannot show (no GPU needed)."""
import os
import re

import pytest

from paper_2609_13846_gb300 import build

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_13846_gb300", "csrc")


def _source(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*", "", re.sub(r"/\*.*?\*/", "", text, flags=re.S))


@pytest.mark.parametrize("name", ["rms_norm.cu", "vocab_loss.cu", "few_loss_f32.cu", "adamw.cu", "layer_host.cuh"])
def test_overlapped_launches_read_coherently_and_wait(name):
    """Each kernel begins before its predecessor has ended: it waits before it touches what that wrote, and reads nothing
    through the read-only path or a pointer declared free of aliases, which may be moved before the wait."""
    text = _source(name)
    assert "__ldg(" not in text and "__restrict__" not in text and "ld.global.nc" not in text
    for body in text.split("__global__")[1:]:
        head = body[:body.index("{")]
        assert "grid_wait();" in body.split("__global__")[0], head


def test_random_roundings_are_not_contracted():
    """The 8-bit codes depend on the last bit of the moments: their sums are scalar and rounded explicitly."""
    text = _source("adamw.cu")
    assert "add.rn.f32x2" not in text and "fma.rn.f32x2" not in text
    assert text.count("= __fadd_rn(m[j") == 2 and text.count("= __fadd_rn(v[j") == 2


def test_lists_of_tensors_are_checked(tmp_path):
    """The native reader refuses what is no list of contiguous CUDA tensors, and names it."""
    import torch

    from paper_2609_13846_gb300 import dtp
    build.build()
    t = torch.zeros(4)
    for args, error, text in ((("params", (t,), 0, None, 1, False), TypeError, "list"), (("params", [3], 0, None, 1, False), TypeError, "params"),
                              (("params", [t], 0, None, 1, False), ValueError, "params must be contiguous CUDA"),
                              (("m", [t], 0, b"", 1, False), ValueError, "m must hold as many"), (("m", [], 0, "x", 1, False), TypeError, "bytes")):
        with pytest.raises(error, match=text):
            dtp._read_list(*args)
    assert dtp._read_list("params", [], 0, None, 1, True) == (b"", b"", b"")
