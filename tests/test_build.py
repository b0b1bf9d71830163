"""The build's order, with the compilers faked: the library is linked even where the binding's module does not compile."""
import os

import pytest

from paper_2506_05413_b200 import build


@pytest.fixture
def faked(tmp_path, monkeypatch):
    def compiled(cmd, **kwargs):
        with open(cmd[cmd.index("-o") + 1], "w") as f:
            f.write("object")
        return build.subprocess.CompletedProcess(cmd, 0, "", "")

    def linked(cmd, **kwargs):
        assert all(os.path.exists(x) for x in cmd if x.endswith(".o"))
        with open(cmd[cmd.index("-o") + 1], "w") as f:
            f.write("library")
        return 0

    monkeypatch.setattr(build, "_nvcc", lambda: "nvcc")
    monkeypatch.setattr(build.subprocess, "run", compiled)
    monkeypatch.setattr(build.subprocess, "check_call", linked)
    monkeypatch.setattr(build, "BUILD", str(tmp_path / "_build"))
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libsmoothrot.so"))
    monkeypatch.setattr(build, "MARSHAL", str(tmp_path / "_marshal.so"))
    return build


def test_the_library_is_linked_where_the_module_does_not_compile(faked, monkeypatch):
    def broken():
        raise RuntimeError("g++ failed on marshal.cpp")

    monkeypatch.setattr(faked, "build_marshal", broken)
    with pytest.raises(RuntimeError, match="marshal"):
        faked.build(force=True)
    assert open(faked.LIB).read() == "library" and not faked.is_current()


def test_both_are_built(faked, monkeypatch):
    def module():
        with open(faked.MARSHAL, "w") as f:
            f.write("module")
        return faked.MARSHAL

    monkeypatch.setattr(faked, "build_marshal", module)
    assert faked.build(force=True) == faked.LIB and os.path.exists(faked.LIB) and faked.is_current()
