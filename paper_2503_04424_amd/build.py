"""Builds libmemdet.so (HIP, gfx950) in-tree next to this file."""
import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmemdet.so")
SOURCES = [os.path.join(CSRC, f) for f in ("memdet.hip", "sequence.hip", "calibrate.hip", "linear.hip", "adamw.hip", "ntk.hip")]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    # packed-FP32 forms are kept out of the generated code on purpose
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-result",
]


def build(verbose: bool = False, extra=()) -> str:
    """Compiles every source, some at a time, and links them."""
    compile_flags = [f for f in FLAGS if f != "-shared"] + list(extra)

    def run(cmd):
        if verbose:
            print(" ".join(cmd))
        subprocess.run(cmd, check=True)

    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, os.path.basename(s) + ".o") for s in SOURCES]
        with ThreadPoolExecutor(max_workers=4) as pool:
            list(pool.map(run, [[HIPCC] + compile_flags + ["-c", "-o", o, s] for s, o in zip(SOURCES, objects)]))
        run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC"] + list(extra) + ["-o", LIB] + objects)
    return LIB


def lib_path() -> str:
    return LIB


if __name__ == "__main__":
    import sys
    print(build(verbose=True, extra=sys.argv[1:]))
