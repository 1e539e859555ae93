"""When the marshalling module is built: for the torch and Python that are there, and not at all without torch -- the C ABI's own
library needs neither.  No compiler is run here."""
import importlib.metadata
import importlib.util
import subprocess

import pytest

from paper_2507_07149_b200 import build


@pytest.fixture
def compiled(monkeypatch):
    """The compiler's calls, in place of the compiler; everything is up to date to begin with."""
    build.build()
    calls = []

    def run(cmd, **kw):
        calls.append(cmd)
        return subprocess.CompletedProcess(cmd, 0, "", "")
    monkeypatch.setattr(build.subprocess, "run", run)
    monkeypatch.setattr(build.subprocess, "check_call", lambda cmd, **kw: calls.append(cmd))
    return calls


def test_an_up_to_date_module_is_left_alone(compiled):
    assert build.build() == build.LIB and not compiled


def test_another_torch_means_another_module(compiled, monkeypatch, tmp_path):
    pytest.importorskip("torch")
    monkeypatch.setattr(build, "MARSHAL_MADE", str(tmp_path / "made"))
    build.build_marshal()
    assert len(compiled) == 1 and build.MARSHAL in compiled[0]
    build.build_marshal()
    assert len(compiled) == 1
    real = importlib.metadata.version
    monkeypatch.setattr(importlib.metadata, "version", lambda name: "9.9.9" if name == "torch" else real(name))
    build.build_marshal()
    assert len(compiled) == 2


def test_without_torch_the_library_is_still_built(compiled, monkeypatch):
    real = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None if name == "torch" else real(name, *a))
    monkeypatch.setattr(build, "_stale", lambda target, deps: True)
    assert build.build() == build.LIB
    assert not any(build.MARSHAL in cmd for cmd in compiled) and any(build.LIB in cmd for cmd in compiled)
