"""Build libtsdp.so in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
import os
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libtsdp.so")
SOURCES = ["tsdp_api.cu", "train_ops.cu"]
DEPS = sorted(f for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))) + ["../../include/tsdp.h"]


def _stale():
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(os.path.join(CSRC, f)) > t for f in SOURCES + DEPS)


def build(force=False, verbose=False):
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    flags = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-diag-suppress", "550", "-Xcompiler", "-fPIC"]
    if verbose:
        flags += ["-Xptxas", "-v"]
    with tempfile.TemporaryDirectory() as tmp:      # the sources side by side, then one library of their objects
        objs = [os.path.join(tmp, f.replace(".cu", ".o")) for f in SOURCES]
        jobs = [subprocess.Popen([nvcc, *flags, "-c", os.path.join(CSRC, f), "-o", o], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
                for f, o in zip(SOURCES, objs)]
        said = [j.communicate()[0] for j in jobs]
        if any(j.returncode for j in jobs):
            raise RuntimeError("nvcc failed:\n" + "".join(said))
        res = subprocess.run([nvcc, *flags[:5], "-shared", "-o", LIB, *objs], capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    if verbose:
        print("".join(said))
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
