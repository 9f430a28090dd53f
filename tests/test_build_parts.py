"""The library and the extension that reads torch tensors are built apart: the first one needs no torch, the second one is built for
one Python and one torch."""
import os
import subprocess

import pytest

from paper_2609_27040_b200 import binding as B
from paper_2609_27040_b200 import build as build_mod


class Commands(list):
    fails = False                                                  # there is no host compiler


@pytest.fixture
def elsewhere(tmp_path, monkeypatch):
    """Products of builds in a folder of the test's, and the commands that would have made them (each leaves an empty product)."""
    ran = Commands()

    class Ran:
        returncode, stdout, stderr = 0, "", ""

    def run(cmd, **_):
        ran.append(cmd)
        if cmd[0] == "g++" and ran.fails:
            raise FileNotFoundError("g++")
        with open(cmd[cmd.index("-o") + 1], "w"):
            return Ran()

    build_mod.build()
    for name in ("LIB", "RESOURCES", "TORCH_CALLS", "TORCH_CALLS_FOR"):
        monkeypatch.setattr(build_mod, name, str(tmp_path / name))
    monkeypatch.setattr(subprocess, "run", run)
    return ran


def test_without_torch_the_library_is_built_all_the_same(elsewhere, monkeypatch, capsys):
    monkeypatch.setattr(build_mod.importlib.util, "find_spec", lambda name: None)
    assert build_mod.build() == build_mod.LIB and os.path.exists(build_mod.LIB)
    assert len(elsewhere) == 1 and "torch is not installed" in capsys.readouterr().err
    with pytest.raises(RuntimeError, match="torch is not installed"):
        build_mod.build_torch_calls()


def test_without_a_host_compiler_the_library_is_built_all_the_same(elsewhere, capsys):
    elsewhere.fails = True
    assert build_mod.build() == build_mod.LIB and os.path.exists(build_mod.LIB) and not os.path.exists(build_mod.TORCH_CALLS)
    assert "not available" in capsys.readouterr().err
    with pytest.raises(RuntimeError, match="cannot be run"):
        build_mod.build_torch_calls()


def test_the_extension_is_built_again_for_another_torch_or_python(elsewhere, monkeypatch):
    import torch
    assert torch.__version__ in build_mod.torch_calls_wanted()
    build_mod.build()
    assert [c[0] == "g++" for c in elsewhere] == [False, True]
    build_mod.build()
    assert len(elsewhere) == 2                                     # as it is
    monkeypatch.setattr(build_mod, "torch_calls_wanted", lambda: "cpython-399 torch 9.9")
    build_mod.build()
    assert len(elsewhere) == 3 and elsewhere[-1][0] == "g++" and build_mod.torch_calls_built_for() == "cpython-399 torch 9.9"
    elsewhere.fails = True                                         # a build that fails leaves nothing that passes for one
    monkeypatch.setattr(build_mod, "torch_calls_wanted", lambda: "cpython-400 torch 9.9")
    build_mod.build()
    assert build_mod.torch_calls_built_for() == ""


def test_an_extension_built_for_another_torch_is_not_loaded(monkeypatch):
    build_mod.build()
    monkeypatch.setattr(B, "_calls", None)
    monkeypatch.setattr(build_mod, "torch_calls_built_for", lambda: "cpython-312 torch 1.0")
    with pytest.raises(RuntimeError, match="built for cpython-312 torch 1.0"):
        B._torch_calls()
    monkeypatch.undo()
    assert B._torch_calls() is not None
