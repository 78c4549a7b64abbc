"""What is built when, with the compilers replaced by ones that fail (no GPU; nothing is compiled)."""
import os

import pytest

from paper_2503_01840_b200 import build


def test_the_library_needs_no_headers_of_python_or_torch(monkeypatch, tmp_path):
    """Where marshal.cpp cannot be compiled the library is built and loaded all the same; only the operators behind it say so."""
    lib = build.build_library()
    ran = []
    real = build.subprocess.run

    class Done:
        returncode, stdout, stderr = 0, "", ""

    def run(cmd, **kw):
        ran.append(cmd)
        if cmd[0] == build.NVCC:
            open(cmd[cmd.index("-o") + 1], "w").close()
            return Done
        return real(cmd, **kw)

    monkeypatch.setattr(build.subprocess, "run", run)
    monkeypatch.setattr(build, "LIB", str(tmp_path / "lib.so"))
    monkeypatch.setattr(build, "OBJ", str(tmp_path / "obj"))
    monkeypatch.setattr(build, "marshal_path", lambda: str(tmp_path / "_marshal.so"))
    monkeypatch.setenv("CXX", "false")
    assert build.build_library() == str(tmp_path / "lib.so") and all(c[0] == build.NVCC for c in ran)
    with pytest.raises(RuntimeError):
        build.build_marshal()
    os.remove(tmp_path / "lib.so")
    with pytest.raises(RuntimeError):
        build.build()
    assert os.path.exists(tmp_path / "lib.so") and not os.path.exists(tmp_path / "_marshal.so")
    monkeypatch.undo()
    assert lib == build.LIB and os.path.getsize(lib) > 0


def test_each_is_built_again_for_its_own_sources(monkeypatch, tmp_path):
    build.build_library()
    monkeypatch.setattr(build, "marshal_path", lambda: str(tmp_path / "_marshal.so"))
    monkeypatch.setattr(build, "LIB", str(tmp_path / "lib.so"))
    newest = {ends: max(os.path.getmtime(os.path.join(build.CSRC, f)) for f in os.listdir(build.CSRC) if f.endswith(ends)) for ends in ((".cu", ".cuh"), ("marshal.cpp",))}
    header = os.path.getmtime(os.path.join(os.path.dirname(build.HERE), "include", "spec_b200.h"))
    for target, ends, check in ((build.LIB, (".cu", ".cuh"), (".cu", ".cuh", ".h")), (build.marshal_path(), ("marshal.cpp",), ("marshal.cpp", ".h"))):
        assert build._stale(target, check)
        open(target, "w").close()
        t = max(newest[ends], header)
        os.utime(target, (t, t))
        assert not build._stale(target, check)
        os.utime(target, (t - 1, t - 1))
        assert build._stale(target, check)


def test_a_module_for_another_torch_or_python_is_not_loaded(monkeypatch):
    here = build.marshal_path()
    assert build.build_marshal() == here and os.path.exists(here)
    with monkeypatch.context() as m:
        m.setattr(build.importlib.metadata, "version", lambda name: "99.1+other")
        other = build.marshal_path()
        assert other != here and build._stale(other, ("marshal.cpp", ".h"))
    with monkeypatch.context() as m:
        m.setattr(build.sysconfig, "get_config_var", lambda name: ".cpython-399.so")
        assert build.marshal_path() not in (here, other)
