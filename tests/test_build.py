"""CPU: the build as a command compiles whether or not anything is out of date (a library built elsewhere, or with another
compiler, may look newer than the sources); as a function it compiles what is out of date."""
import runpy
import subprocess
import types

import pytest

from paper_2609_04098_b200 import build as nvbuild


@pytest.fixture
def refused(monkeypatch):
    """The compiler calls made, none of which is carried out."""
    nvbuild.build()
    calls = []

    def run(cmd, **kw):
        calls.append(cmd)
        return types.SimpleNamespace(returncode=1, stdout="", stderr="")
    monkeypatch.setattr(subprocess, "run", run)
    return calls


def test_the_command_always_compiles(refused, monkeypatch):
    monkeypatch.setattr("sys.argv", ["build"])
    with pytest.raises(RuntimeError, match="nvcc failed"):
        runpy.run_path(nvbuild.__file__, run_name="__main__")
    assert refused and all("-c" in cmd for cmd in refused)


def test_the_function_compiles_nothing_that_is_up_to_date(refused):
    assert nvbuild.build() == nvbuild.LIB
    assert not refused
