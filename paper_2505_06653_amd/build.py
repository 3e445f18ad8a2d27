"""Compile csrc/*.hip for gfx950 into paper_2505_06653_amd/libbof4_hip.so (in-tree, no JIT cache)."""
import glob
import os
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libbof4_hip.so")
SOURCES = sorted(glob.glob(os.path.join(HERE, "csrc", "*.hip")))
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",  # never emit packed-FP32 VALU ops
         "-I", os.path.join(ROOT, "include")]


def build(verbose: bool = False) -> str:
    """All sources side by side (one compiler each), then one link."""
    with tempfile.TemporaryDirectory() as tmp:
        jobs = []
        for src in SOURCES:
            obj = os.path.join(tmp, os.path.basename(src) + ".o")
            cmd = ["hipcc"] + FLAGS + ["-c", "-o", obj, src]
            if verbose:
                print(" ".join(cmd))
            jobs.append((obj, cmd, subprocess.Popen(cmd)))
        failed = [cmd for _, cmd, job in jobs if job.wait() != 0]  # waits for every one of them
        if failed:
            raise subprocess.CalledProcessError(1, failed[0])
        cmd = ["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + [obj for obj, _, _ in jobs]
        if verbose:
            print(" ".join(cmd))
        subprocess.run(cmd, check=True)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
    sys.exit(0)
