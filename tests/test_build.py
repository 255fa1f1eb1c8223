"""What the library's build needs, and what its Python binding does without."""
import os

import pytest

from paper_2607_08779_gb300 import _build, sss


def test_the_library_does_not_wait_for_the_binding(monkeypatch, tmp_path):
    sss.load()
    monkeypatch.setattr(_build, "BINDING", str(tmp_path / "_binding.so"))
    assert _build.up_to_date()

    def fail(*_):
        raise RuntimeError("no compiler")

    monkeypatch.setattr(_build, "build_binding", fail)
    assert _build.build() == _build.LIB


def test_without_the_compiled_part_calls_go_through_ctypes(monkeypatch, tmp_path):
    monkeypatch.setattr(sss, "_fast", None)
    monkeypatch.setattr(_build, "BINDING", str(tmp_path / "_binding.so"))
    monkeypatch.setenv("CXX", "false")
    with pytest.warns(RuntimeWarning, match="ctypes"):
        fast = sss._binding()
    assert fast.page_plan(*[None] * 11) == fast.qk_norm_rope(*[None] * 10) == fast.attention(*[None] * 11) == -1
    assert sss._binding() is fast  # (said once)


def test_a_binding_for_another_torch_is_built_again(monkeypatch, tmp_path):
    sss._binding()
    assert _build.binding_up_to_date()
    other = tmp_path / "binding.stamp"
    other.write_text("another torch")
    monkeypatch.setattr(_build, "STAMP", str(other))
    assert not _build.binding_up_to_date()
    monkeypatch.setattr(_build, "BINDING", str(tmp_path / "_binding.so"))
    _build.build_binding()
    assert _build.binding_up_to_date() and os.path.exists(tmp_path / "_binding.so")
