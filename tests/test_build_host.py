"""When the compiled libraries are taken as built, and what is built without which headers."""
import ctypes
import os

import pytest

from paper_2608_13226_gb300 import build


def test_a_module_of_another_torch_is_not_taken_as_built(monkeypatch):
    build.build()
    assert build.up_to_date()
    monkeypatch.setattr(build, "_torch_id", lambda: "another torch")
    assert not build.up_to_date()
    monkeypatch.undo()
    monkeypatch.setattr(build, "TORCH_MARK", build.TORCH_MARK + ".none")
    assert not build.up_to_date()


def _small(monkeypatch, tmp_path):
    """A library of one small source, in a folder of its own."""
    src = tmp_path / "one.cu"
    src.write_text('extern "C" int one() { return 1; }\n')
    monkeypatch.setattr(build, "BUILD", str(tmp_path))
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libcoverprune.so"))
    monkeypatch.setattr(build, "TORCH_LIB", str(tmp_path / "coverprune_torch.so"))
    monkeypatch.setattr(build, "TORCH_MARK", str(tmp_path / "coverprune_torch.txt"))
    monkeypatch.setattr(build, "_sources", lambda: [str(src)])


def test_the_library_alone_needs_no_torch(monkeypatch, tmp_path):
    """For callers from C: no header of Python or torch has to be there."""
    def none():
        raise ImportError("no torch")
    _small(monkeypatch, tmp_path)
    monkeypatch.setattr(build, "_torch_flags", none)
    monkeypatch.setattr(build, "_torch_id", none)
    assert ctypes.CDLL(build.build(module=False)).one() == 1
    assert build.library_up_to_date() and not os.path.exists(build.TORCH_LIB)


def test_a_module_that_does_not_compile_leaves_the_library(monkeypatch, tmp_path):
    _small(monkeypatch, tmp_path)
    for flags in (lambda: 1 / 0, lambda: (["--no-such-flag"], [])):
        if os.path.exists(build.LIB):
            os.remove(build.LIB)
        monkeypatch.setattr(build, "_torch_flags", flags)
        with pytest.raises(RuntimeError):
            build.build()
        assert build.library_up_to_date() and not build.up_to_date()
