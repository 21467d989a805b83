"""libsp.so does not need what its native Python binding needs."""
import sys

import pytest

import paper_2510_03246_b200
from paper_2510_03246_b200 import api, build


def test_a_binding_that_cannot_be_built_leaves_the_library(monkeypatch, tmp_path):
    build.build()
    for command in (["false"], ["true"], [str(tmp_path / "none")]):          # headers that are missing; a link that fails; no compiler
        monkeypatch.setattr(build, "BINDING", str(tmp_path / "_binding.so"))
        monkeypatch.setattr(build, "_binding_command", lambda out: command)
        monkeypatch.setattr(build, "_binding_link", lambda obj: ["false"])
        with pytest.warns(UserWarning, match="_binding.so"):
            assert build.build() == build.OUT
    monkeypatch.undo()
    assert build.build() == build.OUT and api.lib() is not None


def test_calls_without_the_binding_say_so(monkeypatch):
    monkeypatch.setattr(api, "_native", None)
    monkeypatch.setitem(sys.modules, "paper_2510_03246_b200._binding", None)
    monkeypatch.delattr(paper_2510_03246_b200, "_binding", raising=False)
    with pytest.raises(RuntimeError, match="_binding.so is missing"):
        api._binding()
