"""What the build needs: hipcc for the library of C callers, and more for the extension of the torch entry points."""
import os
import pytest
from paper_2502_04557_amd import build


@pytest.fixture
def commands(monkeypatch, tmp_path):
    """The build up to its commands, which are not run."""
    ran = []
    monkeypatch.setattr(build, "_run", lambda cmd, verbose: ran.append(cmd))
    monkeypatch.setattr(build, "TENSORS", str(tmp_path / "_tensors.so"))
    return ran


def _made(commands):
    return [os.path.basename(c[c.index("-o") + 1]) for c in commands]


def test_the_library_needs_hipcc_alone(commands, monkeypatch, capsys):
    import shutil
    which = shutil.which
    open(build.TENSORS, "w").close()                     # (of other sources: not left beside the new library)
    monkeypatch.setattr(shutil, "which", lambda name, *a, **k: None if name == "g++" else which(name, *a, **k))
    assert build.build_library(verbose=False) == build.LIB
    assert "libsprinter.so" in _made(commands) and "_tensors.so" not in _made(commands) and not os.path.exists(build.TENSORS)
    assert "g++" in capsys.readouterr().out
    monkeypatch.undo()


@pytest.mark.parametrize("gone", ["torch", "Python.h", "extension.h"])
def test_what_the_extension_needs(commands, monkeypatch, gone):
    import sys
    if gone == "torch":
        monkeypatch.setitem(sys.modules, "torch.utils", None)
    else:
        exists = os.path.exists
        monkeypatch.setattr(os.path, "exists", lambda p: not str(p).endswith(gone) and exists(p))
    assert gone in build.tensors_lack()
    build.build_library(verbose=False)
    assert "libsprinter.so" in _made(commands) and "_tensors.so" not in _made(commands)


def test_both_are_built_here(commands):
    assert build.tensors_lack() == ""
    build.build_library(verbose=False)
    assert {"libsprinter.so", "native_bench", "_tensors.so"} <= set(_made(commands))


def test_an_error_of_the_extension_is_one_of_the_build(commands, monkeypatch):
    def run(cmd, verbose):
        if cmd[0] == "g++":
            raise RuntimeError("no")
    monkeypatch.setattr(build, "_run", run)
    with pytest.raises(RuntimeError, match="no"):
        build.build_library(verbose=False)
