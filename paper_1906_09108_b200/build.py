"""Builds libfdg.so in-tree with nvcc for sm_100a.  `python -m paper_1906_09108_b200.build`."""
import os
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libfdg.so")
SOURCES = ["fdg.cu", "norm_ops.cu"]


def _newest_source():
    newest = 0.0
    roots = [CSRC, os.path.join(os.path.dirname(HERE), "include")]
    for root in roots:
        for f in os.listdir(root):
            newest = max(newest, os.path.getmtime(os.path.join(root, f)))
    return newest


def build(force=False, verbose=False):
    if not force and os.path.exists(LIB) and os.path.getmtime(LIB) >= _newest_source():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    flags = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-Xcompiler", "-fPIC"]
    if verbose:
        flags.insert(0, "-Xptxas=-v")
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        runs = [subprocess.Popen([nvcc] + flags + ["-c", "-o", o, os.path.join(CSRC, s)], stdout=subprocess.PIPE,
                                 stderr=subprocess.STDOUT, text=True) for s, o in zip(SOURCES, objects)]
        said = [r.communicate()[0] for r in runs]                     # one process per source, side by side
        if any(r.returncode for r in runs):
            sys.stderr.write("".join(said))
            raise RuntimeError("nvcc failed building libfdg.so")
        if verbose:
            sys.stderr.write("".join(said))
        res = subprocess.run([nvcc] + flags + ["--shared", "-o", LIB] + objects, capture_output=True, text=True)
        if res.returncode != 0:
            sys.stderr.write(res.stdout + res.stderr)
            raise RuntimeError("nvcc failed linking libfdg.so")
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
