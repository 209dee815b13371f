"""Builds libcprune.so (all CUDA sources, sm_100a only) next to this file with nvcc, and _torch_calls.so, the Python module that makes the
operators' calls on torch tensors, with the host compiler."""
from __future__ import annotations

import glob
import importlib.metadata
import os
import subprocess
import sys
import sysconfig
import warnings

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "libcprune.so")
CALLS = os.path.join(HERE, "_torch_calls.so")
BUILD_DIR = os.path.join(HERE, "_build")

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-I", INCLUDE, "-I", CSRC]


def _newest(paths):
    return max(os.path.getmtime(p) for p in paths)


def _calls_for():
    """What _torch_calls.so is built for; the text is compiled into it."""
    try:
        torch_version = importlib.metadata.version("torch")
    except importlib.metadata.PackageNotFoundError:
        torch_version = "unknown"
    return "for torch %s, %s" % (torch_version, sysconfig.get_config_var("SOABI"))


def _calls_command(out):
    import torch
    root = os.path.dirname(torch.__file__)
    include = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"],
               os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include"), INCLUDE]
    libs = os.path.join(root, "lib")
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", *["-I" + p for p in include],
            "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI, '-DBUILT_FOR="%s"' % _calls_for(), os.path.join(CSRC, "torch_calls.cpp"), "-o", out,
            "-L" + libs, "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda", "-Wl,-rpath," + libs]


def _stale(path, deps):
    return not os.path.exists(path) or os.path.getmtime(path) < _newest(deps)


def _calls_stale(headers):
    if _stale(CALLS, [os.path.join(CSRC, "torch_calls.cpp")] + headers):
        return True
    with open(CALLS, "rb") as f:
        return _calls_for().encode() not in f.read()


def _build_calls():
    """The operators' calls in compiled code.  The library loads and works without them (binding.py): what keeps them from being built is told, not raised."""
    tmp = CALLS + ".tmp%d" % os.getpid()
    try:
        subprocess.run(_calls_command(tmp), check=True, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        os.replace(tmp, CALLS)
    except (OSError, ImportError, AttributeError, subprocess.CalledProcessError) as e:
        warnings.warn("_torch_calls.so is not built: %s\n%s" % (e, getattr(e, "output", "") or ""), RuntimeWarning, stacklevel=3)


def build(force: bool = False, verbose: bool = False) -> str:
    srcs, headers = sorted(glob.glob(os.path.join(CSRC, "*.cu"))), glob.glob(os.path.join(INCLUDE, "*.h"))
    lib_deps = srcs + glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.cuh")) + headers
    if force or _stale(LIB, lib_deps):
        _build_lib(srcs, verbose)
    if force or _calls_stale(headers):
        _build_calls()
    return LIB


def _build_lib(srcs, verbose):
    nvcc = os.environ.get("NVCC", "nvcc")
    os.makedirs(BUILD_DIR, exist_ok=True)
    objs, procs = [], []
    for s in srcs:
        o = os.path.join(BUILD_DIR, os.path.basename(s)[:-3] + ".o")
        objs.append(o)
        cmd = [nvcc, *NVCC_FLAGS, "-c", s, "-o", o]
        if verbose:
            cmd.insert(1, "-Xptxas=-v")
        procs.append((s, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = False
    for s, p in procs:
        out, _ = p.communicate()
        if out.strip():
            print(out, file=sys.stderr)
        if p.returncode != 0:
            failed = True
            print("nvcc failed on %s" % s, file=sys.stderr)
    if failed:
        raise RuntimeError("nvcc failed")
    tmp = LIB + ".tmp%d" % os.getpid()
    subprocess.check_call([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-o", tmp, *objs,
                           "-cudart", "static"])
    os.replace(tmp, LIB)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
