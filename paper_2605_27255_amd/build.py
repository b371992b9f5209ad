"""Build the gfx950 HIP library ``libpipo.so`` in-tree.

Every ``csrc/*.hip`` file is compiled with hipcc for gfx950 only, with packed
fp32 arithmetic disabled, and linked into ``paper_2605_27255_amd/libpipo.so``.
"""
from __future__ import annotations

import concurrent.futures as cf
import glob
import os
import re
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "libpipo.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
    "-Wno-unused-result",
]

# k_opd_loss keeps a row of logits in registers across a loop: the constants of
# its few 64-bit exponentials must not be hoisted in front of it (47 registers spilled).
# The compiler reports what its kernels use, and a build in which they spill again says so.
FILE_FLAGS = {"opd_loss.hip": ["-mllvm", "-disable-machine-licm", "-Rpass-analysis=kernel-resource-usage"]}
SPILL_LIMIT = 64        # bytes a thread (the longest bf16 rows' kernel: 20)


def spilled(remarks: str) -> int:
    """The most scratch bytes a thread that the compiler reports for a kernel."""
    return max((int(n) for n in re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", remarks)), default=0)


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, os.path.basename(src) + ".o")
    cmd = [HIPCC, *FLAGS, *FILE_FLAGS.get(os.path.basename(src), []), "-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stdout}\n{r.stderr}")
    if spilled(r.stderr) > SPILL_LIMIT:
        print(f"{os.path.basename(src)}: a kernel spills {spilled(r.stderr)} bytes a thread; it will be slow", file=sys.stderr)
    return obj


def build(jobs: int = 8) -> str:
    os.makedirs(BUILD, exist_ok=True)
    srcs = sorted(glob.glob(os.path.join(CSRC, "*.hip")))
    with cf.ThreadPoolExecutor(max_workers=jobs) as ex:
        objs = list(ex.map(_compile, srcs))
    tmp = LIB + ".tmp"
    r = subprocess.run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", tmp],
                       capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(int(sys.argv[1]) if len(sys.argv) > 1 else 8))
