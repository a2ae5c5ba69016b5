"""Build libdsim.so (HIP, gfx950) and the operators' Python binding in-tree.

    python -m paper_2111_05426_amd.build

Every translation unit of the library is compiled as HIP for gfx950 with FMA
contraction off (the simulator's fp64 results must not depend on contraction
choices) and packed-fp32 instructions disabled.  The binding (_ops.so) is
host C++ against torch's headers, linked to libdsim.so beside it.
"""
import glob
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libdsim.so")
BINDING = os.path.join(HERE, "_ops.so")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")

FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
         "-ffp-contract=off", "-fno-fast-math", "-fno-gpu-rdc", "-fvisibility=hidden",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wall", "-Wno-unused-function", "-I", INCLUDE]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cpp")) + glob.glob(os.path.join(CSRC, "*.hip")))


def binding_sources():
    return sorted(glob.glob(os.path.join(HERE, "binding", "*.cpp")))


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)


def _build_library(hipcc, verbose):
    # one compiler a source, at most as many at once as MAX_JOBS allows
    jobs = max(1, min(8, int(os.environ.get("MAX_JOBS") or os.cpu_count() or 1)))
    flags = [f for f in FLAGS if f != "-shared"]
    with tempfile.TemporaryDirectory() as tmp, ThreadPoolExecutor(jobs) as pool:
        objects = [os.path.join(tmp, os.path.basename(s) + ".o") for s in sources()]
        list(pool.map(lambda so: _run([hipcc] + flags + ["-x", "hip", "-c", so[0], "-o", so[1]], verbose),
                      zip(sources(), objects)))
        _run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC"] + objects + ["-o", LIB + ".tmp"], verbose)
    os.replace(LIB + ".tmp", LIB)


def _torch_root():
    """torch's folder, or None; torch itself is not imported."""
    spec = importlib.util.find_spec("torch")
    return os.path.dirname(spec.origin) if spec and spec.origin else None


def _build_binding(verbose):
    """The operators' binding; without torch's headers or a C++ compiler it is
    left out, and the operators' Python calls raise ImportError."""
    root, cxx = _torch_root(), os.environ.get("CXX", "g++")
    lacks = ("torch's headers" if not root or not os.path.isdir(os.path.join(root, "include", "torch")) else
             "a C++ compiler (%s)" % cxx if not shutil.which(cxx.split()[0]) else None)
    if os.path.exists(BINDING):
        os.remove(BINDING)   # (one of another library's)
    if lacks:
        print("the operators' Python binding is not built: it needs %s" % lacks, file=sys.stderr)
        return
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    cmd = cxx.split() + ["-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-Wall",
                         "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1", "-I", INCLUDE,
                         "-isystem", os.path.join(root, "include"),
                         "-isystem", os.path.join(root, "include", "torch", "csrc", "api", "include"),
                         "-isystem", os.path.join(rocm, "include"), "-isystem", sysconfig.get_paths()["include"]]
    cmd += binding_sources() + ["-o", BINDING + ".tmp", "-L", HERE, "-l:" + os.path.basename(LIB), "-Wl,-rpath,$ORIGIN",
                                "-L", os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10",
                                "-lc10_hip"]
    _run(cmd, verbose)
    os.replace(BINDING + ".tmp", BINDING)


def build(verbose=False):
    _build_library(os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), verbose)
    _build_binding(verbose)
    return LIB


if __name__ == "__main__":
    build(verbose="-v" in sys.argv)
    print(LIB)
