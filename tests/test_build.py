"""The build's steps with stand-ins for the compilers (nothing is compiled)."""
import subprocess

import pytest


def test_the_library_does_not_need_the_binding(monkeypatch, tmp_path):
    """Where the native binding does not compile (no g++, no headers of torch) the library is built, and the error is
    raised."""
    from paper_1507_04296_amd import build
    out = tmp_path / "libgorila.so"

    def no_binding():
        raise RuntimeError("g++ failed for binding.cpp")

    def link(cmd, **kw):
        open(cmd[cmd.index("-o") + 1], "w").write("linked")
        return subprocess.CompletedProcess(cmd, 0, "", "")

    monkeypatch.setattr(build, "BUILD_DIR", str(tmp_path))
    monkeypatch.setattr(build, "OUT", str(out))
    monkeypatch.setattr(build, "_compile", lambda src: src + ".o")
    monkeypatch.setattr(build, "_compile_binding", no_binding)
    monkeypatch.setattr(build.subprocess, "run", link)
    with pytest.raises(RuntimeError, match="binding.cpp"):
        build.build()
    assert out.read_text() == "linked"
