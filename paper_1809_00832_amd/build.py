"""Compile the HIP library (csrc/*.hip) for gfx950 into libtreelstm.so next to this file."""
import os
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
SOURCES = ("treelstm", "attend_f32", "attend_bf16", "attend_f16", "decoder")
SRC = os.path.join(HERE, "csrc", "treelstm.hip")
LIB = os.path.join(HERE, "libtreelstm.so")


def build(verbose: bool = False) -> str:
    flags = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-I", os.path.join(ROOT, "include"), "-I", os.path.join(HERE, "csrc")]
    if verbose:
        flags.insert(0, "-Rpass-analysis=kernel-resource-usage")
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, name + ".o") for name in SOURCES]
        compilers = [subprocess.Popen(["hipcc", *flags, "-c", "-o", obj, os.path.join(HERE, "csrc", name + ".hip")])
                     for name, obj in zip(SOURCES, objects)]
        failed = [name for name, c in zip(SOURCES, compilers) if c.wait() != 0]
        if failed:
            raise RuntimeError("hipcc failed: " + ", ".join(failed))
        subprocess.run(["hipcc", "--offload-arch=gfx950", "-fPIC", "-shared", "-o", LIB, *objects], check=True)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
