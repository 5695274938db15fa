"""Build libscoot.so for gfx950, in-tree.

Every ``csrc/*.hip`` file is compiled by hipcc for --offload-arch=gfx950 with
packed-fp32 instructions disabled; host-only ``csrc/*.cpp`` files by g++.  The
shared library lands next to this file, where the binding loads it from, and
beside it the module of binding/kv_torch.cpp, which calls it with torch tensors.
"""
import concurrent.futures as cf
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OUT_DIR = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libscoot.so")
MODULE = os.path.join(HERE, "_kv_torch.so")
ARCH = "gfx950"

HIP_FLAGS = ["-O3", "-fPIC", "-std=c++17", f"--offload-arch={ARCH}",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-I", os.path.join(ROOT, "include"), "-I", CSRC]
CXX_FLAGS = ["-O3", "-fPIC", "-std=c++17", "-fopenmp-simd", "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _hipcc():
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("hipcc not found")


def _compile(src, hipcc):
    obj = os.path.join(OUT_DIR, os.path.basename(src) + ".o")
    if src.endswith(".hip"):
        cmd = [hipcc, *HIP_FLAGS, "-c", src, "-o", obj]
    else:
        cmd = ["g++", *CXX_FLAGS, "-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    return obj


def _module_needs():
    """What the module is compiled against and this machine lacks: torch's or Python's headers."""
    import sysconfig
    try:
        import torch
    except ImportError:
        return "torch"
    for path in (os.path.join(os.path.dirname(torch.__file__), "include", "ATen", "ATen.h"),
                 os.path.join(sysconfig.get_paths()["include"], "Python.h")):
        if not os.path.exists(path):
            return path
    return None


def _build_module():
    """The Python module over torch's tensors (host code only).  libscoot.so does without it: where its headers are
    missing it is left out, and only the calls that need it raise.  Returns whether it was built."""
    lacks = _module_needs()
    if lacks:
        if os.path.exists(MODULE):
            os.remove(MODULE)  # of another build of the library
        print(f"{os.path.basename(MODULE)} (calls of the cache operators from torch) not built: {lacks} is missing", file=sys.stderr)
        return False
    import sysconfig

    import torch
    base = os.path.dirname(torch.__file__)
    tmp = MODULE + ".tmp"
    cmd = ["g++", "-O2", "-fPIC", "-std=c++17", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-I", os.path.join(base, "include"), "-I", os.path.join(base, "include", "torch", "csrc", "api", "include"),
           "-I", sysconfig.get_paths()["include"], os.path.join(HERE, "binding", "kv_torch.cpp"), "-o", tmp,
           "-L", os.path.join(base, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, MODULE)
    return True


def build(jobs=None, verbose=False):
    """Compile every source, link libscoot.so and the module over it.  Always rebuilds."""
    os.makedirs(OUT_DIR, exist_ok=True)
    hipcc = _hipcc()
    srcs = sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".hip", ".cpp")))
    jobs = jobs or min(len(srcs), max(1, min(16, os.cpu_count() or 1)))
    with cf.ThreadPoolExecutor(jobs) as ex:
        module = ex.submit(_build_module)
        objs = list(ex.map(lambda s: _compile(s, hipcc), srcs))
    tmp = LIB + ".tmp"
    cmd = [hipcc, "-shared", "-fPIC", f"--offload-arch={ARCH}", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    both = module.result()
    if verbose:
        print(f"built {LIB} and {MODULE}" if both else f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
