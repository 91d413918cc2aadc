"""How the library is built: the commands, seen by a compiler that only writes down what it is asked for."""
import os

import pytest

from paper_2508_20407_amd import build as hip_build


@pytest.fixture
def commands(tmp_path, monkeypatch):
    """hipcc's command lines, in order, of builds that compile nothing."""
    log, fake = tmp_path / "log", tmp_path / "hipcc"
    fake.write_text(f'#!/bin/sh\necho "$*" >> "{log}"\n')
    fake.chmod(0o755)
    monkeypatch.setenv("PATH", f"{tmp_path}{os.pathsep}{os.environ['PATH']}")
    monkeypatch.setattr(hip_build, "LIB_PATH", str(tmp_path / "lib.so"))
    return lambda: [line.split() for line in log.read_text().splitlines()]


def test_extra_flags_reach_compiles_and_link(commands):
    hip_build.build(extra=["-Lsomewhere", "-lsomething", "-DNAME=1"])
    lines = commands()
    compiles, links = [c for c in lines if "-c" in c], [c for c in lines if "-c" not in c]
    assert len(compiles) == 2 and len(links) == 1 and lines[-1] is links[0]
    for line in lines:
        assert {"-Lsomewhere", "-lsomething", "-DNAME=1", "--offload-arch=gfx950", "-fPIC"} <= set(line)
    # a library is asked for behind the objects that want it
    link = links[0]
    assert link.index("-lsomething") > max(i for i, x in enumerate(link) if x.endswith(".o") and link[i - 1] != "-o")
    assert "-shared" in link and link[link.index("-o") + 1] == hip_build.LIB_PATH


def test_all_device_code_is_compiled_without_packed_fp32(commands):
    hip_build.build()
    for line in commands():
        if "-c" in line:
            assert " ".join(line).count("-Xclang -target-feature -Xclang -packed-fp32-ops") == 1
