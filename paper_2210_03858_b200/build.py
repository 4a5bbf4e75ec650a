"""Builds the library in-tree: csrc/*.cu -> libbcq_b200.so (sm_100a only), csrc/binding.c and csrc/binding_torch.cpp -> the
extension modules _bcq_call and _tensor_call, whose file names carry the interpreter's ABI tag.

Only _tensor_call needs torch (with CUDA): its headers, and the C++ ABI of its libraries, so its file name carries torch's version
too, and it is left out where there is no torch.  The library and _bcq_call are what callers of include/bcq.h need."""
from __future__ import annotations

import contextlib
import glob
import importlib.util
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
OBJ_DIR = os.path.join(HERE, "_build")

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC"]


def _torch():
    """(directory, version, CUDA version or None) of the installed torch, without importing it; None if there is none."""
    spec = importlib.util.find_spec("torch")
    if spec is None or not spec.origin:
        return None
    root, about = os.path.dirname(spec.origin), {}
    try:
        with open(os.path.join(root, "version.py")) as f:
            exec(f.read(), about)
    except OSError:
        return None
    return root, str(about["__version__"]), about.get("cuda")


def tensor_call_path():
    """Where the extension module _tensor_call for the installed torch is, built or not; None without a torch that has CUDA."""
    torch = _torch()
    if torch is None or torch[2] is None:
        return None
    return os.path.join(HERE, "_tensor_call.torch-%s%s" % (torch[1], sysconfig.get_config_var("EXT_SUFFIX")))


def _sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _headers():
    return glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.cuh")) + [os.path.join(os.path.dirname(HERE), "include", "bcq.h")]


def _older(path, sources) -> bool:
    return not os.path.exists(path) or any(os.path.getmtime(p) > os.path.getmtime(path) for p in sources)


def _library_is_stale() -> bool:
    sources = _sources() + _headers() + [os.path.join(CSRC, "binding.c")]
    return _older(LIB, sources) or _older(CALL, sources)


def _tensor_call_is_stale() -> bool:
    path = tensor_call_path()
    return path is not None and _older(path, [os.path.join(CSRC, "binding_torch.cpp")] + _headers())


def is_stale() -> bool:
    return _library_is_stale() or _tensor_call_is_stale()


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
    out = tensor_call_path()
    root = os.path.dirname(torch.__file__)
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    lib = os.path.join(root, "lib")
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI]
    cmd += ["-I" + p for p in (sysconfig.get_paths()["include"],)]
    cmd += ["-isystem" + p for p in (os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
                                     os.path.join(cuda, "include"))]
    cmd += [os.path.join(CSRC, "binding_torch.cpp"), "-o", out + ".tmp", "-L" + lib, "-Wl,-rpath," + lib, "-ltorch_python", "-ltorch",
            "-ltorch_cuda", "-ltorch_cpu", "-lc10_cuda", "-lc10", "-ldl"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("g++ failed for binding_torch.cpp:\n" + r.stderr)
    os.replace(out + ".tmp", out)


def _build_cuda(verbose: bool):
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

    with ThreadPoolExecutor(max_workers=4) as ex:
        objs = list(ex.map(compile_one, _sources()))
    cmd = [nvcc, "-shared", "-o", LIB + ".tmp"] + objs + ["-gencode", "arch=compute_100a,code=sm_100a"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stderr)
    os.replace(LIB + ".tmp", LIB)
    _build_binding()


def build_library(force: bool = False, verbose: bool = False) -> str:
    with ThreadPoolExecutor(max_workers=1) as ex:
        binding = ex.submit(_build_tensor_binding) if _tensor_call_is_stale() or (force and tensor_call_path()) else None
        if force or _library_is_stale():
            _build_cuda(verbose)
        if binding is not None:
            binding.result()
    if tensor_call_path():
        for other in set(glob.glob(os.path.join(HERE, "_tensor_call*.so"))) - {tensor_call_path()}:  # for another torch
            with contextlib.suppress(FileNotFoundError):  # (another process may have removed it)
                os.remove(other)
    return LIB


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv))
