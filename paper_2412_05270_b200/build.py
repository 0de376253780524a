"""Builds libapollo.so (hand-written CUDA for sm_100a) in-tree with nvcc."""
from __future__ import annotations

import importlib.util
import os
import subprocess
from pathlib import Path

PKG = Path(__file__).resolve().parent
CSRC = PKG / "csrc"
LIB = PKG / "libapollo.so"
LIB_DEBUG = PKG / "libapollo_debug.so"      # the same sources with -DAPOLLO_DEBUG: index checks inside the kernels of contexts
SOURCES = ["apollo_api.cu", "kernels_basic.cu", "kernels_tensor.cu", "apollo_static.cu", "kernels_adamw.cu",
           "apollo_muon.cu", "kernels_muon.cu", "kernels_embedding.cu", "kernels_logprob.cu", "kernels_adamw_list.cu",
           "kernels_adjust.cu"]
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden",
]


def _stale(lib: Path = LIB) -> bool:
    if not lib.exists():
        return True
    built = lib.stat().st_mtime
    deps = list(CSRC.glob("*")) + [PKG.parent / "include" / "apollo.h", Path(__file__)]
    return any(p.stat().st_mtime > built for p in deps)


def marshal_path() -> Path:
    """The binding's extension (csrc/marshal.cpp: what it asks of tensors) for the Python and the torch that are running; one built for others has
    another name (their tensors lie otherwise in memory)."""
    import sysconfig

    import torch
    return PKG / f"_marshal.{sysconfig.get_config_var('SOABI')}.torch-{torch.__version__}.so"


def build_marshal(force: bool = False) -> Path:
    """Compiles the Python extension that reads tensors for the binding (against torch's headers; torch is loaded first)."""
    src, path = CSRC / "marshal.cpp", marshal_path()
    if not force and path.exists() and path.stat().st_mtime >= max(src.stat().st_mtime, Path(__file__).stat().st_mtime):
        return path
    import sysconfig

    import torch
    from torch.utils import cpp_extension
    tmp = path.with_name(f"{path.name}.{os.getpid()}.tmp")
    include = [f"-I{p}" for p in cpp_extension.include_paths()] + [f"-I{sysconfig.get_paths()['include']}"]
    libs = [f"-L{p}" for p in cpp_extension.library_paths()] + ["-lc10", "-ltorch_cpu", "-ltorch_python"]
    out = subprocess.run([os.environ.get("CXX", "g++"), "-shared", "-fPIC", "-O2", "-std=c++17", "-fvisibility=hidden", "-w",
                          f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", *include, str(src), "-o", str(tmp), *libs],
                         stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if out.returncode != 0:
        print(out.stdout)
        raise RuntimeError("g++ failed on marshal.cpp")
    os.replace(tmp, path)
    return path


def build_library(force: bool = False, verbose: bool = False, debug: bool = False) -> Path:
    """Compiles the library in-tree, with nvcc alone, and then, where torch is installed, the binding's extension.  debug=True builds
    libapollo_debug.so: the kernels of contexts (apollo_create, apollo_muon_create) check the index range of their global loads and stores and
    report a violation through the status word (apollo_status returns APOLLO_ERR_INTERNAL) instead of making the access; the stateless
    entry points have no status word, and their kernels no checks."""
    lib = _compile(force, verbose, debug)
    if importlib.util.find_spec("torch") is not None:
        build_marshal(force)
    return lib


def _compile(force: bool, verbose: bool, debug: bool) -> Path:
    lib = LIB_DEBUG if debug else LIB
    if not force and not _stale(lib):
        return lib
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    objs = []
    obj_dir = PKG / ("_build/debug" if debug else "_build")
    obj_dir.mkdir(parents=True, exist_ok=True)
    flags = NVCC_FLAGS + (["-DAPOLLO_DEBUG"] if debug else [])
    procs = []
    for src in SOURCES:
        obj = obj_dir / (src + ".o")
        cmd = [nvcc, *flags, "-c", str(CSRC / src), "-o", str(obj)]
        if verbose:
            cmd.insert(1, "-Xptxas=-v")
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(str(obj))
    for src, p in procs:
        out, _ = p.communicate()
        if verbose or p.returncode != 0:
            print(out)
        if p.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}")
    tmp = lib.with_suffix(f".{os.getpid()}.tmp")
    subprocess.run([nvcc, "-shared", "-o", str(tmp), *objs, "-Xcompiler", "-fvisibility=hidden"], check=True)
    os.replace(tmp, lib)
    return lib


if __name__ == "__main__":
    import sys
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv, debug="--debug" in sys.argv))
