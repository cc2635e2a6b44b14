"""Build libptd.so in-tree from csrc/*.cu with nvcc for sm_103a (one -gencode, parallel TUs), and
the Python binding's call module _ptdcall.so from csrc/pycall.cpp."""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
OUT = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libptd.so")
CALLS = os.path.join(PKG, "_ptdcall.so")
CALLS_FOR = os.path.join(OUT, "ptdcall_for")   # what the call module was compiled against
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC"]


def nvcc() -> str:
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libptd.so")
    return exe


def _sources():
    return sorted(f for f in os.listdir(CSRC) if f.endswith(".cu"))


def _compile(src: str) -> str:
    obj = os.path.join(OUT, src[:-3] + ".o")
    cmd = [nvcc(), *ARCH, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"nvcc failed on {src}:\n{r.stdout}\n{r.stderr}")
    return obj


def _calls_for() -> str:
    """What the call module has to be compiled against anew for: it reads torch's tensors by the layout of one version."""
    import torch

    return f"torch {torch.__version__}, C++11 ABI {int(torch._C._GLIBCXX_USE_CXX11_ABI)}, {sysconfig.get_config_var('SOABI')}"


def _compile_calls() -> None:
    import torch

    root = os.path.dirname(os.path.abspath(torch.__file__))   # its headers and libraries: the module looks at its tensors
    include, lib = os.path.join(root, "include"), os.path.join(root, "lib")
    tmp = CALLS + ".tmp"
    cmd = [shutil.which("g++") or "g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f'-DPTD_TORCH_VERSION="{torch.__version__}"',
           "-isystem", include, "-isystem", os.path.join(include, "torch", "csrc", "api", "include"),
           "-I", sysconfig.get_paths()["include"], os.path.join(CSRC, "pycall.cpp"), "-o", tmp, "-ldl", "-L", lib,
           f"-Wl,-rpath,{lib}", "-ltorch_python", "-ltorch_cpu", "-lc10"]
    if os.path.exists(CALLS_FOR):   # (written behind the module: one left half made is made again)
        os.remove(CALLS_FOR)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed on pycall.cpp:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, CALLS)
    with open(CALLS_FOR, "w") as f:
        f.write(_calls_for())


def _calls_fit() -> bool:
    """Whether the call module there is was compiled for this torch and this interpreter."""
    if not os.path.exists(CALLS_FOR):
        return False
    with open(CALLS_FOR) as f:
        return f.read() == _calls_for()


def build(force: bool = False) -> str:
    """Compile every CUDA source and link the shared library (and the call module); returns its path."""
    os.makedirs(OUT, exist_ok=True)
    srcs = _sources()
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [
        os.path.join(os.path.dirname(PKG), "include", "ptd.h")]
    newest = max(os.path.getmtime(d) for d in deps)
    fresh = [not force and os.path.exists(f) and os.path.getmtime(f) >= newest for f in (LIB, CALLS)]
    if all(fresh):
        if not _calls_fit():
            _compile_calls()
        return LIB
    with cf.ThreadPoolExecutor(max_workers=min(8, len(srcs))) as ex:
        calls = ex.submit(_compile_calls)
        objs = list(ex.map(_compile, srcs))
    tmp = LIB + ".tmp"
    cmd = [nvcc(), *ARCH, "-shared", "-cudart", "static", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    calls.result()   # (the library is there whatever becomes of the module)
    return LIB


if __name__ == "__main__":
    print(build(force=True))
