"""What a build needs: the library and the oracle need no torch, and no C++
compiler besides hipcc's; the tensor binding is left out where they are missing."""
import importlib.util
import os
import shutil

import pytest

import __graft_entry__ as entry

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def made(monkeypatch, tmp_path):
    """The things that build() makes, none of them compiled; the binding goes
    to a folder of the test's."""
    spec = importlib.util.spec_from_file_location("lib_build", os.path.join(ROOT, "paper_2509_18172_amd", "build.py"))
    lib = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(lib)
    names = []

    class Oracle:
        @staticmethod
        def build():
            names.append("oracle")

    def run(cmd, **kwargs):
        names.append("binding")
        open(cmd[cmd.index("-o") + 1], "w").write("new")
        return type("Done", (), dict(returncode=0))
    monkeypatch.setattr(lib, "build", lambda: names.append("library"))
    monkeypatch.setattr(lib, "build_probe", lambda: names.append("probe"))
    monkeypatch.setattr(lib, "binding_path", lambda: str(tmp_path / "binding.so"))
    monkeypatch.setattr(lib.subprocess, "run", run)
    monkeypatch.setattr(entry, "_build_module", lambda path: Oracle if "oracle" in path else lib)
    (tmp_path / "binding.so").write_text("old")
    names.append(tmp_path / "binding.so")
    return names


def test_build(made):
    entry.build()
    assert made[1:] == ["library", "probe", "binding", "oracle"] and made[0].read_text() == "new"


@pytest.mark.parametrize("missing", ["torch", "compiler"])
def test_build_without_what_only_the_binding_needs(made, monkeypatch, capsys, missing):
    if missing == "torch":
        find = importlib.util.find_spec
        monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))
        real = __import__

        def no_torch(name, *args, **kwargs):
            if name.split(".")[0] == "torch":
                raise ImportError("no torch")
            return real(name, *args, **kwargs)
        monkeypatch.setattr("builtins.__import__", no_torch)
    else:
        monkeypatch.setattr(shutil, "which", lambda name: None)
    entry.build()
    assert made[1:] == ["library", "probe", "oracle"]
    assert not made[0].exists()  # an older build's would not fit the library
    assert "binding" in capsys.readouterr().err
