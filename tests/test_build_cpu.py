"""When the library is built anew: by what changed, with a compiler that only writes down what it is asked for."""
import os
from pathlib import Path

import pytest


@pytest.fixture()
def tree(tmp_path, monkeypatch):
    from paper_2503_06671_b200 import build

    csrc, include = tmp_path / "csrc", tmp_path / "include"
    csrc.mkdir(), include.mkdir()
    for name, text in (("one.cu", '#include "both.cuh"\n'), ("two.cu", "\n"), ("both.cuh", "\n")):
        (csrc / name).write_text(text)
    (include / "api.h").write_text("\n")
    for name, value in (("CSRC", csrc), ("INCLUDE", include), ("LIB_DIR", tmp_path / "lib"), ("OBJ_DIR", tmp_path / "lib" / "obj"),
                        ("LIB", tmp_path / "lib" / "lib.so"), ("NVCC_FLAGS", ["-O3"])):
        monkeypatch.setattr(build, name, value)
    for f in [*csrc.iterdir(), *include.iterdir()]:
        os.utime(f, (1e9, 1e9))
    calls = []

    def compiler(cmd):
        Path(cmd[cmd.index("-o") + 1]).write_text(" ".join(cmd))
        calls.append([Path(c).name for c in cmd if c.endswith(".cu")] or ["link"])

    monkeypatch.setattr(build, "_nvcc", lambda: "nvcc")
    monkeypatch.setattr(build.subprocess, "check_call", compiler)

    def built(**o):
        calls.clear()
        build.build(**o)
        return sorted(sum(calls, []))

    return build, csrc, built, monkeypatch


def test_what_is_compiled(tree):
    build, csrc, built, monkeypatch = tree
    assert built() == ["link", "one.cu", "two.cu"]
    assert built() == [] and built(verbose=True) == []
    os.utime(csrc / "both.cuh")
    later = build.LIB.stat().st_mtime + 10
    os.utime(csrc / "both.cuh", (later, later))
    assert built() == ["link", "one.cu"]
    assert built(force=True) == ["link", "one.cu", "two.cu"]


def test_other_flags_compile_everything(tree):
    build, csrc, built, monkeypatch = tree
    built()
    monkeypatch.setattr(build, "NVCC_FLAGS", ["-O3", "-DX"])
    assert build.needs_build() and built() == ["link", "one.cu", "two.cu"]
    assert "-DX" in build.LIB.read_text() and len(list(build.OBJ_DIR.glob("*.o"))) == 2
    assert not build.needs_build() and built() == []
    (csrc / "two.cu").unlink()
    assert build.needs_build() and built() == ["link"] and len(list(build.OBJ_DIR.glob("*.o"))) == 1
