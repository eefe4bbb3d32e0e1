"""The native marshalling module is used only with the interpreter and the torch that it was compiled for (CPU)."""
import os
import subprocess
import sys
import types

import pytest

from paper_2603_04135_b200 import binding as B
from paper_2603_04135_b200 import build

NAME = "paper_2603_04135_b200._marshal"


def test_built_module_names_what_it_was_built_for():
    if not os.path.exists(build.MARSHAL):
        pytest.skip("not built")
    import importlib
    assert importlib.import_module(NAME).built_for == build.built_for()
    assert B._load_native() is sys.modules[NAME]


@pytest.mark.parametrize("built_for", [None, "cpython-39 torch 1.0"])
def test_module_of_another_torch_is_left_alone(monkeypatch, built_for):
    used = []
    other = types.ModuleType(NAME)
    other.bind = lambda *a: used.append(a)
    if built_for is not None:
        other.built_for = built_for
    monkeypatch.setitem(sys.modules, NAME, other)
    monkeypatch.setattr(sys.modules["paper_2603_04135_b200"], "_marshal", other, raising=False)
    native = B._load_native()
    assert native is not other and not used
    assert native.token_logprobs(1, 2, 3) is None and native.linear_i8() is None     # nothing is the plain case: Python's checks


def test_module_of_another_torch_is_built_again(monkeypatch, tmp_path):
    ran = []
    monkeypatch.setattr(build, "MARSHAL", str(tmp_path / "_marshal.so"))
    monkeypatch.setattr(build, "MARSHAL_STAMP", str(tmp_path / "marshal.stamp"))

    def compiler(cmd, **k):
        ran.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()
        return subprocess.CompletedProcess(cmd, 0, "", "")
    monkeypatch.setattr(build.subprocess, "run", compiler)
    build.build_marshal()
    build.build_marshal()
    assert len(ran) == 1                                             # up to date
    monkeypatch.setattr(build, "built_for", lambda: "cpython-313 torch 9.9")
    build.build_marshal()
    build.build_marshal()
    assert len(ran) == 2 and any("torch 9.9" in a for a in ran[1])
    os.remove(build.MARSHAL_STAMP)                                   # built by who knows what
    build.build_marshal()
    assert len(ran) == 3
