"""What build() compiles, with the compilers replaced by one that writes an
empty file."""

import sys

import pytest

from paper_2301_09830_amd import build


@pytest.fixture
def compilers(monkeypatch, tmp_path):
    ran = []

    class Compiler:
        returncode = 0

        def __init__(self, cmd, **_):
            ran.append(cmd)
            open(cmd[cmd.index("-o") + 1], "w").close()

        def communicate(self):
            return "", ""

    def run(cmd, **kw):
        p = Compiler(cmd)
        p.stderr = ""
        return p

    monkeypatch.setattr(build.subprocess, "Popen", Compiler)
    monkeypatch.setattr(build.subprocess, "run", run)
    monkeypatch.setattr(build, "hipcc", lambda: "hipcc")
    monkeypatch.setattr(build, "LIB", str(tmp_path / "liboptcc.so"))
    monkeypatch.setattr(build, "LAYERS", str(tmp_path / "_layers.so"))
    return ran


def test_the_library_builds_without_torch(compilers, monkeypatch, tmp_path):
    """The C interface does not need torch, and neither does its build."""
    monkeypatch.setitem(sys.modules, "torch", None)       # import torch fails
    assert build.build() == str(tmp_path / "liboptcc.so")
    assert sorted(p.name for p in tmp_path.iterdir()) == ["liboptcc.so"]
    assert [c[0] for c in compilers] == ["hipcc"] * 3     # two sources and the link


def test_the_binding_builds_where_torch_is(compilers, tmp_path):
    pytest.importorskip("torch")
    build.build()
    assert sorted(p.name for p in tmp_path.iterdir()) == ["_layers.so", "liboptcc.so"]
    assert sorted(c[0] for c in compilers) == ["g++"] + ["hipcc"] * 3
