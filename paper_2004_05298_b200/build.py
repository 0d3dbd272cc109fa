"""Compile the CUDA library in-tree: csrc/*.cu -> paper_2004_05298_b200/libdef_b200.so.

nvcc cross-compiles for sm_100a without a GPU.  The library links the CUDA runtime
statically, so it loads (and its host-side validation runs) on a machine without a
driver; only launching needs a B200.
"""
import os
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "libdef_b200.so")
SOURCES = ["def_api.cu", "def_train_api.cu", "def_block_api.cu", "def_feed_api.cu", "def_orthogonal_api.cu"]
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-cudart", "static",
]


def _nvcc():
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    raise RuntimeError("nvcc not found")


def _inputs():
    files = [os.path.join(CSRC, f) for f in sorted(os.listdir(CSRC))]
    files += [os.path.join(INCLUDE, f) for f in sorted(os.listdir(INCLUDE))]
    return files


def needs_build():
    if not os.path.exists(LIB):
        return True
    built = os.path.getmtime(LIB)
    return any(os.path.getmtime(f) > built for f in _inputs())


def build(force=False, verbose=False):
    """Run nvcc if the library is missing or older than its sources; returns its path."""
    if not force and not needs_build():
        return LIB
    nvcc = [_nvcc(), *NVCC_FLAGS]
    with tempfile.TemporaryDirectory(prefix="def_b200_") as objs:   # one nvcc per source, side by side: 145 s instead of 213
        runs = []
        for src in SOURCES:
            obj = os.path.join(objs, src + ".o")
            cmd = nvcc + ["-I", INCLUDE] + (["-Xptxas", "-v"] if verbose else []) + ["-c", os.path.join(CSRC, src), "-o", obj]
            runs.append((obj, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        outs = [(run.communicate()[0], run.returncode) for _, run in runs]
        said = "".join(out for out, _ in outs)
        failed = any(rc for _, rc in outs)
        tmp = LIB + ".tmp.%d" % os.getpid()
        if not failed:
            link = subprocess.run(nvcc + ["-shared"] + [obj for obj, _ in runs] + ["-o", tmp],
                                  stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
            said, failed = said + link.stdout, link.returncode != 0
    if verbose or failed:
        sys.stderr.write(said)
    if failed:
        if os.path.exists(tmp):
            os.remove(tmp)
        raise RuntimeError("nvcc failed:\n" + said)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
