"""Build libtlinattn.so for gfx950 with hipcc (in-tree, next to this file)."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB_PATH = os.path.join(HERE, "libtlinattn.so")
SRC = os.path.join(HERE, "csrc", "tlinattn.hip")
# the paged cache: a translation unit of its own, linked behind the first
PAGED_SRC = os.path.join(HERE, "csrc_paged", "paged.hip")

# Packed-fp32 VALU instructions are switched off for all device code.
HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-shared", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
]


def build(verbose: bool = False, extra=()) -> str:
    """The library's path.  extra: flags for every compile and for the link."""
    inc = ["-I", os.path.join(ROOT, "include"), "-I", os.path.join(HERE, "csrc"), "-I", os.path.join(HERE, "csrc_paged")]
    with tempfile.TemporaryDirectory() as tmp:
        objs, jobs = [], []
        for src in (SRC, PAGED_SRC):
            objs.append(os.path.join(tmp, os.path.basename(src) + ".o"))
            cmd = ["hipcc", *(f for f in HIPCC_FLAGS if f != "-shared"), *extra, *inc, "-c", src, "-o", objs[-1]]
            if verbose:
                print(" ".join(cmd), flush=True)
            jobs.append(subprocess.Popen(cmd, stdout=subprocess.DEVNULL, stderr=subprocess.PIPE, text=True))
        results = [(job.communicate()[1], job.returncode) for job in jobs]      # both run on side by side
        link = ["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-Wno-unused-command-line-argument", *objs, *extra, "-o", LIB_PATH]
        if all(rc == 0 for _, rc in results):
            if verbose:
                print(" ".join(link), flush=True)
            res = subprocess.run(link, capture_output=True, text=True)
            results.append((res.stderr, res.returncode))
    # the host pass does not know the device-only target feature and says so: harmless
    err = "\n".join(l for text, _ in results for l in text.splitlines() if "packed-fp32-ops" not in l)
    if any(rc != 0 for _, rc in results):
        raise RuntimeError("hipcc failed:\n" + err)
    if verbose and err.strip():
        print(err, file=sys.stderr)
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose=True, extra=sys.argv[1:]))
