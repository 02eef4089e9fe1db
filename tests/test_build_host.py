"""When the compiled libraries are taken as built, and what is built without which headers."""
from paper_2608_13226_gb300 import build


def test_a_module_of_another_torch_is_not_taken_as_built(monkeypatch):
    build.build()
    assert build.up_to_date()
    monkeypatch.setattr(build, "_torch_id", lambda: "another torch")
    assert not build.up_to_date()
    monkeypatch.undo()
    monkeypatch.setattr(build, "TORCH_MARK", build.TORCH_MARK + ".none")
    assert not build.up_to_date()
