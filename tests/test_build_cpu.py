"""What the build needs and when it builds again."""
import os

import pytest

from paper_2605_24058_b200 import build, lordba


def test_the_library_does_without_the_python_module(monkeypatch, capsys):
    """A C user has nvcc and no headers of torch or Python."""
    build.build_library()

    def missing(force=False):
        raise RuntimeError("torch/extension headers not found")

    monkeypatch.setattr(build, "build_binding", missing)
    assert build.build_library() == build.LIB
    assert "headers not found" in capsys.readouterr().err


def test_the_module_is_built_again_for_another_torch(monkeypatch):
    build.build_binding()
    calls = []

    class Done:
        returncode, stdout, stderr = 0, "", ""

    def compile_only_in_name(cmd, **kw):
        calls.append(cmd)
        return Done()

    monkeypatch.setattr(build.subprocess, "run", compile_only_in_name)
    monkeypatch.setattr(build.os, "replace", lambda a, b: calls.append((a, b)))
    build.build_binding()
    assert not calls                                              # nothing changed: nothing is built
    monkeypatch.setattr(build, "binding_made_for", lambda: "Python 3.0, torch 0.1")
    build.build_binding()
    assert calls and any("torch 0.1" in part for part in calls[0])
    for a, _ in calls[1:]:
        if os.path.exists(a):
            os.remove(a)


def test_a_module_of_another_torch_is_refused(monkeypatch):
    build.build_library()
    build.build_binding()
    monkeypatch.setattr(lordba, "_block", None)
    assert lordba._native().made_for == build.binding_made_for()
    monkeypatch.setattr(lordba, "_block", None)
    monkeypatch.setattr(build, "binding_made_for", lambda: "Python 3.0, torch 0.1")
    with pytest.raises(RuntimeError, match="torch 0.1"):
        lordba._native()
