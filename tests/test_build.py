"""Builds that run at the same time do not meet in a file: nvcc is a script here that notes what it is to write."""
import os
import stat

import pytest

from paper_2601_20357_b200 import build

FAKE = """#!/bin/sh
while [ $# -gt 0 ]; do if [ "$1" = -o ]; then out="$2"; fi; shift; done
echo "$out" >> "{log}"
if [ -n "$FAIL" ]; then echo broken; exit 1; fi
echo made > "$out"
"""


@pytest.fixture
def fake(tmp_path, monkeypatch):
    log, nvcc, pkg = tmp_path / "log", tmp_path / "nvcc", tmp_path / "pkg"
    pkg.mkdir()
    nvcc.write_text(FAKE.format(log=log))
    nvcc.chmod(nvcc.stat().st_mode | stat.S_IXUSR)
    monkeypatch.setenv("NVCC", str(nvcc))
    monkeypatch.setattr(build, "PKG_DIR", str(pkg))
    monkeypatch.setattr(build, "CSRC", str(pkg))
    monkeypatch.setattr(build, "LIB_PATH", str(pkg / "lib.so"))
    return log, pkg


def test_two_builds_share_no_file_but_the_finished_library(fake):
    log, pkg = fake
    written = []
    for _ in range(2):
        assert build.build(force=True) == build.LIB_PATH
        written.append(set(log.read_text().split()))
        log.unlink()
    assert len(written[0]) == len(build.SOURCES) + 1 and not written[0] & written[1]
    assert build.LIB_PATH not in written[0] | written[1]          # it appears whole
    assert os.listdir(pkg) == ["lib.so"] and (pkg / "lib.so").read_text() == "made\n"


def test_a_failed_build_leaves_the_library_as_it_was(fake, monkeypatch):
    log, pkg = fake
    build.build(force=True)
    (pkg / "lib.so").write_text("before")
    monkeypatch.setenv("FAIL", "1")
    with pytest.raises(RuntimeError, match="broken"):
        build.build(force=True)
    assert os.listdir(pkg) == ["lib.so"] and (pkg / "lib.so").read_text() == "before"
