"""The host side of the paged cache's entry points (argument checks, workspaces, frequencies: everything that returns before the
first HIP call) under AddressSanitizer and UndefinedBehaviorSanitizer.  Device code is compiled as usual and never runs here."""
import os
import shutil

import pytest

from test_sanitizers import ENV, NATIVE, ROOT, SAN, run


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not found")
def test_paged_host_side_under_address_and_undefined_behaviour_sanitizers(tmp_path):
    obj, drv, exe = (str(tmp_path / n) for n in ("paged_asan.o", "driver.o", "paged_api_asan"))
    package = os.path.join(ROOT, "paper_2508_20407_amd")
    inc = ["-I", os.path.join(ROOT, "include"), "-I", os.path.join(package, "csrc"), "-I", os.path.join(package, "csrc_paged")]
    # sanitizers on the host pass only: each -fsanitize= directly behind its own -Xarch_host
    run(["hipcc", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-command-line-argument",
         "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
         "-Xarch_host", "-fno-sanitize-recover=undefined", *inc,
         "-c", os.path.join(package, "csrc_paged", "paged.hip"), "-o", obj], cwd=str(tmp_path))
    clang = os.path.join(os.path.dirname(os.path.realpath(shutil.which("hipcc"))), "..", "lib", "llvm", "bin", "clang")
    if not os.path.exists(clang):
        clang = "/opt/rocm/lib/llvm/bin/clang"
    run([clang, "-O1", "-g", *SAN, *inc, "-c", os.path.join(NATIVE, "paged_api_driver.c"), "-o", drv])
    # link only (no device compile on this line): the sanitizer runtimes for the host objects
    run(["hipcc", "--offload-arch=gfx950", "-fno-gpu-sanitize", "-fsanitize=address,undefined", obj, drv, "-o", exe], cwd=str(tmp_path))
    r = run([exe], env=dict(ENV, ASAN_OPTIONS=ENV["ASAN_OPTIONS"].replace("detect_leaks=1", "detect_leaks=0")), timeout=300)
    assert "paged api driver ok" in r.stdout and "runtime error" not in r.stderr
