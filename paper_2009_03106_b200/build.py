"""Build libdpclip.so in-tree with nvcc for sm_100a (no JIT cache involved)."""
from __future__ import annotations

import glob
import importlib.metadata
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "libdpclip.so")
MARSHAL = os.path.join(HERE, "_marshal.so")                # Python module: arguments of the transformer-block calls
MARSHAL_KEY = os.path.join(HERE, "build", "marshal.key")   # what _marshal.so was built for
LIB_DEBUG = os.path.join(HERE, "libdpclip_debug.so")       # -DDPCLIP_DEBUG: range-checked accesses

NVCC_FLAGS = ["-std=c++17", "-O3", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
              "-Xcompiler", "-fPIC", "-I" + INCLUDE, "-I" + CSRC]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _stale(lib: str = LIB) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    deps = glob.glob(os.path.join(CSRC, "*")) + glob.glob(os.path.join(INCLUDE, "*.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def _object_stale(obj: str, dep: str) -> bool:
    """Whether an object file is older than its source or any header it was compiled from (nvcc -MD writes the list)."""
    if not (os.path.exists(obj) and os.path.exists(dep)):
        return True
    with open(dep) as f:
        names = f.read().replace("\\\n", " ").split(":", 1)[1].split()
    t = os.path.getmtime(obj)
    own = [n for n in names if os.path.abspath(n).startswith(os.path.dirname(HERE))]
    return any(not os.path.exists(n) or os.path.getmtime(n) > t for n in own)


def _marshal_built_for() -> str:
    """What the module is compiled against beside its sources: the C++ interfaces of torch and of the interpreter."""
    return f"torch {importlib.metadata.version('torch')}, Python {sys.version}"


def _marshal_stale() -> bool:
    if not (os.path.exists(MARSHAL) and os.path.exists(MARSHAL_KEY)):
        return True
    with open(MARSHAL_KEY) as f:
        if f.read() != _marshal_built_for():
            return True
    t = os.path.getmtime(MARSHAL)
    return any(os.path.getmtime(d) > t for d in (os.path.join(CSRC, "marshal.cpp"), os.path.join(INCLUDE, "dpclip.h")))


def _start_marshal(force: bool):
    """Start compiling csrc/marshal.cpp, where the module is older or was built for another torch or Python; None where there is nothing to do."""
    src = os.path.join(CSRC, "marshal.cpp")
    if not force and not _marshal_stale():
        return None
    import sysconfig

    import torch
    root = os.path.dirname(torch.__file__)
    tmp = MARSHAL + f".tmp{os.getpid()}"
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I" + INCLUDE, "-I" + sysconfig.get_paths()["include"],
           "-isystem", os.path.join(root, "include"), "-isystem", os.path.join(root, "include", "torch", "csrc", "api", "include"),
           "-isystem", os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include"), src, "-L" + os.path.join(root, "lib"),
           "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda", "-o", tmp]
    return cmd, tmp, subprocess.Popen(cmd)


def _finish_marshal(started) -> None:
    if started is None:
        return
    cmd, tmp, p = started
    if p.wait() != 0:
        raise subprocess.CalledProcessError(p.returncode, cmd)
    os.replace(tmp, MARSHAL)
    os.makedirs(os.path.dirname(MARSHAL_KEY), exist_ok=True)
    with open(MARSHAL_KEY, "w") as f:
        f.write(_marshal_built_for())


def build(force: bool = False, verbose: bool = False, debug: bool = False) -> str:
    """Compile every .cu under csrc/, each to an object of its own and all at once, and link one shared library; and the Python module that
    marshals arguments to it.  Returns the library's path.
    debug=True builds libdpclip_debug.so (range-checked accesses that set DPCLIP_ERR_RANGE and skip) beside it."""
    lib = LIB_DEBUG if debug else LIB
    marshal = _start_marshal(force and not debug)
    if not force and not _stale(lib):
        _finish_marshal(marshal)
        return lib
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    objects = os.path.join(HERE, "build", "debug" if debug else "release")
    os.makedirs(objects, exist_ok=True)
    flags = NVCC_FLAGS + (["-DDPCLIP_DEBUG"] if debug else []) + (["-Xptxas", "-v"] if verbose else [])
    running, objs = [], []
    for src in sources():
        name = os.path.splitext(os.path.basename(src))[0]
        obj, dep = os.path.join(objects, name + ".o"), os.path.join(objects, name + ".d")
        objs.append(obj)
        if force or verbose or _object_stale(obj, dep):
            tmp = f"{obj}.tmp{os.getpid()}.o"
            cmd = [nvcc] + flags + ["-c", src, "-o", tmp, "-MD", "-MF", dep]
            running.append((cmd, tmp, obj, subprocess.Popen(cmd)))
    for cmd, tmp, obj, p in running:
        if p.wait() != 0:
            raise subprocess.CalledProcessError(p.returncode, cmd)
        os.replace(tmp, obj)
    tmp = lib + f".tmp{os.getpid()}"
    subprocess.check_call([nvcc] + NVCC_FLAGS + ["-shared"] + objs + ["-o", tmp])
    os.replace(tmp, lib)
    _finish_marshal(marshal)
    return lib


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, debug="--debug" in sys.argv))
