"""Builds the library in-tree: csrc/*.cu -> libbcq_b200.so (sm_100a only), csrc/binding.c and csrc/binding_torch.cpp -> the
extension modules _bcq_call and _tensor_call, whose file names carry the interpreter's ABI tag."""
from __future__ import annotations

import glob
import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libbcq_b200.so")
# the tag keeps another interpreter version from importing an extension that was not built for it
CALL = os.path.join(HERE, "_bcq_call" + sysconfig.get_config_var("EXT_SUFFIX"))
TENSOR_CALL = os.path.join(HERE, "_tensor_call" + sysconfig.get_config_var("EXT_SUFFIX"))
OBJ_DIR = os.path.join(HERE, "_build")

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC"]


def _sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _deps():
    return _sources() + glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.cuh")) + \
        [os.path.join(CSRC, "binding.c"), os.path.join(CSRC, "binding_torch.cpp"), os.path.join(os.path.dirname(HERE), "include", "bcq.h")]


def is_stale() -> bool:
    built = (LIB, CALL, TENSOR_CALL)
    if not all(os.path.exists(p) for p in built):
        return True
    t = min(os.path.getmtime(p) for p in built)
    return any(os.path.getmtime(p) > t for p in _deps())


def _build_binding():
    cmd = [os.environ.get("CC", "gcc"), "-O2", "-fPIC", "-shared", "-I" + sysconfig.get_paths()["include"],
           os.path.join(CSRC, "binding.c"), "-o", CALL + ".tmp", "-ldl"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("gcc failed for binding.c:\n" + r.stderr)
    os.replace(CALL + ".tmp", CALL)
    untagged = os.path.join(HERE, "_bcq_call.so")  # of an older tree: any interpreter would import it
    if os.path.exists(untagged):
        os.remove(untagged)


def _build_tensor_binding():
    import torch
    root = os.path.dirname(torch.__file__)
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    lib = os.path.join(root, "lib")
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI]
    cmd += ["-I" + p for p in (sysconfig.get_paths()["include"],)]
    cmd += ["-isystem" + p for p in (os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
                                     os.path.join(cuda, "include"))]
    cmd += [os.path.join(CSRC, "binding_torch.cpp"), "-o", TENSOR_CALL + ".tmp", "-L" + lib, "-Wl,-rpath," + lib, "-ltorch_python", "-ltorch",
            "-ltorch_cuda", "-ltorch_cpu", "-lc10_cuda", "-lc10", "-ldl"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("g++ failed for binding_torch.cpp:\n" + r.stderr)
    os.replace(TENSOR_CALL + ".tmp", TENSOR_CALL)


def build_library(force: bool = False, verbose: bool = False) -> str:
    if not force and not is_stale():
        return LIB
    nvcc = os.environ.get("NVCC", "nvcc")
    os.makedirs(OBJ_DIR, exist_ok=True)

    def compile_one(src):
        obj = os.path.join(OBJ_DIR, os.path.basename(src)[:-3] + ".o")
        cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-c", src, "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("nvcc failed for %s:\n%s" % (src, r.stderr))
        if verbose:
            sys.stderr.write(r.stderr)
        return obj

    with ThreadPoolExecutor(max_workers=5) as ex:
        binding = ex.submit(_build_tensor_binding)
        objs = list(ex.map(compile_one, _sources()))
        binding.result()
    cmd = [nvcc, "-shared", "-o", LIB + ".tmp"] + objs + ["-gencode", "arch=compute_100a,code=sm_100a"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stderr)
    os.replace(LIB + ".tmp", LIB)
    _build_binding()
    return LIB


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv))
