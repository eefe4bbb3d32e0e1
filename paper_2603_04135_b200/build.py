"""Builds libdppo.so (sm_100a, nvcc) and the binding's argument marshalling (_marshal.so, host compiler) in-tree.
`python -m paper_2603_04135_b200.build`."""
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OBJ = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libdppo.so")
MARSHAL = os.path.join(PKG, "_marshal.so")
MARSHAL_STAMP = os.path.join(OBJ, "marshal.stamp")       # what MARSHAL was built for

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC]


def _nvcc():
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    raise RuntimeError("nvcc not found")


def sources():
    return sorted(f for f in os.listdir(CSRC) if f.endswith(".cu"))


def _stale(target, deps):
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def build_library(force=False, verbose=False):
    """Compile every csrc/*.cu and link libdppo.so next to this file.  Returns the library path."""
    os.makedirs(OBJ, exist_ok=True)
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))]
    headers.append(os.path.join(ROOT, "include", "dppo.h"))
    nvcc = _nvcc()
    jobs = []
    for src in sources():
        s = os.path.join(CSRC, src)
        o = os.path.join(OBJ, src[:-3] + ".o")
        if force or _stale(o, [s] + headers):
            jobs.append([nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-c", s, "-o", o])

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("nvcc failed: %s\n%s\n%s" % (" ".join(cmd), r.stdout, r.stderr))
        if verbose:
            sys.stderr.write(r.stderr)

    with ThreadPoolExecutor(max_workers=max(1, min(8, len(jobs) or 1))) as ex:
        list(ex.map(run, jobs))
    objs = [os.path.join(OBJ, src[:-3] + ".o") for src in sources()]
    if force or jobs or _stale(LIB, objs):
        run([nvcc, "-shared", "-gencode", "arch=compute_100a,code=sm_100a", "-o", LIB] + objs)
    return LIB


def built_for():
    """The interpreter and torch whose layouts a module compiled now relies on."""
    import torch
    return "%s torch %s" % (sys.implementation.cache_tag, torch.__version__)


def build_marshal(force=False):
    """Compile csrc/marshal.cpp against this interpreter's and torch's headers.  Returns the module's path."""
    src = os.path.join(CSRC, "marshal.cpp")
    stamp = None
    if os.path.exists(MARSHAL_STAMP):
        with open(MARSHAL_STAMP) as f:
            stamp = f.read()
    if not force and stamp == built_for() and not _stale(MARSHAL, [src, os.path.join(ROOT, "include", "dppo.h")]):
        return MARSHAL
    import sysconfig

    import torch
    tdir = os.path.dirname(torch.__file__)
    tlib = os.path.join(tdir, "lib")
    cuda = os.path.dirname(os.path.dirname(_nvcc())) if os.path.sep in _nvcc() else "/usr/local/cuda"
    inc = [os.path.join(tdir, "include"), os.path.join(tdir, "include", "torch", "csrc", "api", "include"),
           os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-I" + os.path.join(ROOT, "include"),
           "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI), '-DDPPO_BUILT_FOR="%s"' % built_for()]
    cmd += [x for p in inc for x in ("-isystem", p)]
    cmd += [src, "-o", MARSHAL, "-L" + tlib, "-Wl,-rpath," + tlib, "-ltorch_python", "-ltorch_cpu", "-lc10_cuda", "-lc10"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("host compiler failed: %s\n%s\n%s" % (" ".join(cmd), r.stdout, r.stderr))
    os.makedirs(OBJ, exist_ok=True)
    with open(MARSHAL_STAMP, "w") as f:
        f.write(built_for())
    return MARSHAL


if __name__ == "__main__":
    print(build_marshal(force="--force" in sys.argv))
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv))
