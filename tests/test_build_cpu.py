"""The library builds and loads without the short way of its calls (csrc/calls.cpp), and a _calls.so of
another torch is left alone."""

import importlib.metadata
import importlib.util
import os
import sys
import types

import pytest

from paper_2504_05346_b200 import build as B


@pytest.fixture
def aside(tmp_path, monkeypatch):
    """A built library, and a stale _calls.so in a folder of its own."""
    B.build()
    calls = tmp_path / "_calls.so"
    calls.write_bytes(b"stale")
    monkeypatch.setattr(B, "CALLS", str(calls))
    monkeypatch.setattr(B, "CALLS_STAMP", str(tmp_path / "calls_stamp.txt"), raising=False)
    return calls


@pytest.mark.parametrize("command", [["/no/such/compiler"], [sys.executable, "-c", "raise SystemExit(1)"]],
                         ids=["no compiler", "an error"])
def test_a_failing_compiler_leaves_the_library(aside, monkeypatch, capsys, command):
    monkeypatch.setattr(B, "_calls_command", lambda *a: command)
    assert B.build() == B.LIB and os.path.exists(B.LIB)
    assert not aside.exists()
    assert "long way" in capsys.readouterr().err


def test_the_library_needs_no_torch(aside, monkeypatch, capsys):
    def missing(name, *a):
        raise importlib.metadata.PackageNotFoundError(name)

    monkeypatch.setattr(importlib.metadata, "version", missing)
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None)
    assert B.build() == B.LIB
    assert not aside.exists() and "torch" in capsys.readouterr().err


def test_built_once(aside, monkeypatch):
    """What is there is compiled again only for other sources; it is never written over in place."""
    monkeypatch.setattr(B, "_calls_command",
                        lambda out: [sys.executable, "-c", "open(%r, 'w').write('new')" % out])
    before = os.stat(aside).st_ino
    with open(aside) as held:
        B.build()
        assert held.read() == "stale"
    assert aside.read_text() == "new" and os.stat(aside).st_ino != before
    first = os.stat(aside).st_ino
    monkeypatch.setattr(B, "_calls_command", None)
    monkeypatch.setattr(B, "nvcc_path", None)
    B.build()
    assert os.stat(aside).st_ino == first


@pytest.mark.parametrize("built_for, taken", [(None, False), ("torch 1.0.0, python 3.12", False),
                                              ("here", True)])
def test_calls_of_another_torch_are_not_bound(monkeypatch, built_for, taken):
    import torch
    import paper_2504_05346_b200 as T
    from paper_2504_05346_b200 import binding

    B.build()
    lib = T.load_library()
    bound = []
    fake = types.ModuleType("paper_2504_05346_b200._calls")
    fake.bind = lambda *a: bound.append(a)
    if built_for is not None:
        fake.built_for = "torch %s, python %d.%d" % ((torch.__version__,) + sys.version_info[:2]) \
            if built_for == "here" else built_for
    monkeypatch.setattr(T, "_calls", fake, raising=False)
    monkeypatch.setitem(sys.modules, "paper_2504_05346_b200._calls", fake)
    monkeypatch.setattr(binding, "_calls", None)
    binding._bind_calls(lib)
    assert (binding._calls is fake) == taken and len(bound) == taken
