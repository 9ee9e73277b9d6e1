"""The build: the library of the C ABI needs hipcc alone; the compiled side of the Python calls is built where its prerequisites are there."""
import importlib.util
import os
import shutil

from paper_2504_15364_amd import build as kd_build


def test_a_missing_prerequisite_is_named(monkeypatch, tmp_path):
    assert kd_build.calls_lack() is None
    with monkeypatch.context() as m:
        m.setattr(importlib.util, "find_spec", lambda name, *a: None)
        assert "torch" in kd_build.calls_lack()
    with monkeypatch.context() as m:
        m.setattr(shutil, "which", lambda name, *a, **k: None)
        assert "g++" in kd_build.calls_lack()
    with monkeypatch.context() as m:
        m.setattr(kd_build.sysconfig, "get_paths", lambda *a: {"include": str(tmp_path)})
        assert "Python.h" in kd_build.calls_lack()


def test_the_library_is_built_without_them(monkeypatch, tmp_path, capsys):
    calls, done = tmp_path / "_calls.so", []
    calls.write_bytes(b"of an earlier build")

    class Compiled:
        returncode = 0

        def __init__(self, cmd, **kw):
            done.append(cmd)

        def communicate(self):
            return "", None

    monkeypatch.setattr(kd_build.subprocess, "Popen", Compiled)
    monkeypatch.setattr(kd_build.subprocess, "run", lambda cmd, check: done.append(cmd))
    monkeypatch.setattr(kd_build, "CALLS", str(calls))
    monkeypatch.setattr(kd_build, "calls_lack", lambda: "torch is not installed")
    assert kd_build.build() == kd_build.LIB
    assert all(cmd[0] == "hipcc" for cmd in done) and len(done) == len(kd_build.SOURCES) + 1
    # one that stands for other sources is not left beside the new library
    assert not os.path.exists(calls)
    assert "torch is not installed" in capsys.readouterr().err
