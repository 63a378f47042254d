"""Build libfiona.so for gfx950 in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
SRCS = [os.path.join(HERE, "csrc", "fiona.hip"), os.path.join(HERE, "csrc", "rescale.hip"),
        os.path.join(HERE, "csrc", "rotate.hip"), os.path.join(HERE, "csrc", "microbench.hip"),
        os.path.join(HERE, "csrc", "ntt_check.hip"), os.path.join(HERE, "csrc", "append.hip"),
        os.path.join(HERE, "csrc", "attention.hip"), os.path.join(HERE, "csrc", "adapter.hip")]
OUT = os.path.join(HERE, "libfiona.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

# Packed fp32 instructions are disabled for all HIP code (the kernels are
# integer; this keeps the compiler from forming them anywhere).
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(HERE, "csrc")]


def build(verbose: bool = False) -> str:
    tmp = OUT + ".tmp%d" % os.getpid()
    cmd = [HIPCC] + FLAGS + SRCS + ["-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + r.stderr)
    if verbose and r.stderr:
        print(r.stderr)
    os.replace(tmp, OUT)
    return OUT


if __name__ == "__main__":
    print(build(verbose=True))
