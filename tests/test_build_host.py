"""The build on the CPU: what makes the extension out of date, and that a build that fails leaves what was there."""
import os
import subprocess
import sys

import pytest


@pytest.fixture
def build(tmp_path, monkeypatch):
    from paper_2609_32712_b200 import build as b
    monkeypatch.setattr(b, "NATIVE", str(tmp_path / "_native.so"))
    monkeypatch.setattr(b, "LIB", str(tmp_path / "libmala.so"))
    monkeypatch.setattr(b, "_build_library", lambda verbose: open(b.LIB, "w").close())
    return b


def _compiles(b, monkeypatch, text, code=0):
    """The compiler's place: writes `text` where its output goes, and ends with `code`."""
    calls = []

    def command(out):
        calls.append(out)
        return [sys.executable, "-c", f"import sys; open(sys.argv[1], 'w').write({text!r}); sys.exit({code})", out]
    monkeypatch.setattr(b, "_native_command", command)
    return calls


def test_built_once_for_a_torch_and_an_interpreter(build, monkeypatch):
    calls = _compiles(build, monkeypatch, "one")
    build.build()
    build.build()
    assert len(calls) == 1 and open(build.NATIVE).read() == "one"
    for name, value in (("__version__", "0.0.other"), ("__file__", "/elsewhere/torch/__init__.py")):
        import torch
        with monkeypatch.context() as m:
            m.setattr(torch, name, value)
            n = len(calls)
            build.build()
            build.build()
            assert len(calls) == n + 1
    n = len(calls)
    monkeypatch.setattr(build.sysconfig, "get_config_var", lambda key: "cpython-other" if key == "SOABI" else None)
    build.build()
    assert len(calls) == n + 1


def test_a_build_that_fails_leaves_the_old_file(build, monkeypatch):
    _compiles(build, monkeypatch, "good")
    build.build()
    _compiles(build, monkeypatch, "part of", code=1)
    with pytest.raises(subprocess.CalledProcessError):
        build.build(force=True)
    folder = os.path.dirname(build.NATIVE)
    assert open(build.NATIVE).read() == "good" and not [f for f in os.listdir(folder) if "tmp" in f]
    calls = _compiles(build, monkeypatch, "better")
    build.build(force=True)
    assert len(calls) == 1 and open(build.NATIVE).read() == "better"


def test_a_file_without_its_record_is_built_again(build, monkeypatch):
    calls = _compiles(build, monkeypatch, "one")
    open(build.NATIVE, "w").write("from before")
    build.build()
    assert len(calls) == 1 and open(build.NATIVE).read() == "one"
