"""The binding's native reader of tensor lists belongs to one torch: another rebuilds it, and does not load it (no GPU needed)."""
import os

import pytest

from paper_2609_13846_gb300 import build, dtp


@pytest.fixture
def other_torch(monkeypatch, tmp_path):
    """The module as another torch left it: newer than its sources."""
    build.build()
    record = tmp_path / "tensor_lists.for"
    record.write_text("torch 2.1.0, cpython-312, x86_64")
    monkeypatch.setattr(build, "LISTS_FOR", str(record))
    monkeypatch.setattr(dtp, "_tensor_lists", None)
    return record


def test_a_module_of_another_torch_is_not_loaded(other_torch):
    with pytest.raises(RuntimeError, match=r"torch 2\.1\.0.*build it again"):
        dtp._read_list("params", [], 0, None, 1, True)
    other_torch.unlink()                  # nor one whose versions nobody wrote down
    with pytest.raises(RuntimeError, match="build it again"):
        dtp._read_list("params", [], 0, None, 1, True)


def test_a_module_of_another_torch_is_built_again(other_torch, monkeypatch):
    built = []
    monkeypatch.setattr(build, "_build_lists", lambda: built.append(1))
    build.build()
    assert built == [1]
    other_torch.write_text(build.versions())
    build.build()
    assert built == [1] and os.path.exists(build.LISTS)


def test_what_is_built_is_loaded():
    build.build()
    assert build.lists_versions() == build.versions()
    assert dtp._read_list("params", [], 0, None, 1, True) == (b"", b"", b"")


def test_versions_are_counted_for_lists_alone():
    import torch
    build.build()
    dtp._read_list("params", [], 0, None, 1, True)
    t = torch.zeros(3)
    before = t._version
    dtp._tensor_lists.written([t, None], [])
    assert t._version == before + 1
    with pytest.raises(TypeError, match="lists"):
        dtp._tensor_lists.written((t,))
    with torch.inference_mode():
        u = torch.zeros(3)
    dtp._tensor_lists.written([u])
