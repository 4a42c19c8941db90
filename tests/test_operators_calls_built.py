"""CPU tests of when the compiled calls are used: beside the torch and Python that they were built for, and no other."""
import subprocess
import sys

import pytest
import torch

import paper_2605_25550_amd as dm
from paper_2605_25550_amd import build as B


@pytest.fixture
def calls(monkeypatch):
    dm.lib()
    if dm._CALLS is None:
        pytest.skip("the compiled calls are not built")
    real = dm._CALLS
    monkeypatch.setattr(dm, "_CALLS", None)
    return real


class Stand:
    """A module in the compiled calls' place."""

    def __init__(self, **kw):
        self.bound = False
        self.__dict__.update(kw)

    def bind(self, *args):
        self.bound = True


def in_its_place(monkeypatch, module):
    monkeypatch.setitem(sys.modules, dm.__name__ + "._marshal", module)
    monkeypatch.setattr(dm, "_marshal", module, raising=False)
    dm._bind_calls(dm.lib())


def test_the_module_says_what_it_was_built_for(calls):
    assert calls.BUILT_FOR == B.marshal_target()
    assert torch.__version__ in calls.BUILT_FOR and hex(sys.hexversion) in calls.BUILT_FOR


def test_the_same_torch_and_python(calls, monkeypatch):
    m = Stand(BUILT_FOR=B.marshal_target())
    in_its_place(monkeypatch, m)
    assert m.bound and dm._CALLS is m


@pytest.mark.parametrize("built_for", [None, "", "torch 1.0", "other python"])
def test_another_torch_or_python(calls, monkeypatch, built_for):
    m = Stand() if built_for is None else Stand(BUILT_FOR=B.marshal_target().replace("Python", "Python 9")
                                                if built_for == "other python" else built_for)
    in_its_place(monkeypatch, m)
    assert not m.bound and dm._CALLS is None


def test_another_torchs_version(calls, monkeypatch):
    monkeypatch.setattr(torch, "__version__", "2.99.0")
    dm._bind_calls(dm.lib())
    assert dm._CALLS is None


@pytest.mark.parametrize("how", ["no compiler", "no headers"])
def test_a_build_without_them(monkeypatch, tmp_path, how):
    """The library is built all the same, and no module of an earlier build stays beside it."""
    lib, old = tmp_path / "lib.so", tmp_path / "_marshal.so"
    old.write_bytes(b"of an earlier build")
    real = subprocess.run

    def run(cmd, **kw):
        if cmd[0] == "g++":
            if how == "no compiler":
                raise FileNotFoundError(2, "No such file or directory: 'g++'")
            return real([sys.executable, "-c", "raise SystemExit('Python.h: No such file')"], **kw)
        (tmp_path / "lib.so.tmp").write_bytes(b"linked")
        return real([sys.executable, "-c", ""], **kw)
    for name, value in (("SOURCES", []), ("OBJDIR", str(tmp_path)), ("LIB", str(lib)), ("MARSHAL", str(old))):
        monkeypatch.setattr(B, name, value)
    monkeypatch.setattr(B.subprocess, "run", run)
    with pytest.warns(UserWarning, match="(?s)compiled calls were not built.*No such file"):
        assert B.build() == str(lib)
    assert lib.read_bytes() == b"linked" and not old.exists()
