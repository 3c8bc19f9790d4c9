"""Compile the CUDA sources into paper_2310_11453_b200/libbitlinear_b200.so for sm_100a, and the argument
marshalling of the attention operators and the 8-bit layers into paper_2310_11453_b200/_marshal.so.

nvcc cross-compiles without a GPU.  The library links the static CUDA runtime and nothing else,
so it loads in any process (with or without torch) on a box that has the driver; _marshal is a Python
module against torch's C++ interface.  The library needs nvcc alone and is built whatever becomes of _marshal, which also
takes torch's and Python's headers: where those are missing, the attention operators of the Python binding say so when
they are called, and the rest works.
"""
import glob
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libbitlinear_b200.so")
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17",
         "-Xcompiler", "-fPIC", "-fmad=true"]


OBJ = os.path.join(HERE, "_build")
MARSHAL_SRC = os.path.join(CSRC, "marshal.cpp")
MARSHAL = os.path.join(HERE, "_marshal.so")


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _stale(target, deps) -> bool:
    deps = deps + [os.path.join(HERE, "..", "include", "bitlinear.h")]
    return not os.path.exists(target) or any(os.path.getmtime(d) > os.path.getmtime(target) for d in deps)


def _marshal_command():
    import torch
    root = os.path.dirname(torch.__file__)
    inc, libs = os.path.join(root, "include"), os.path.join(root, "lib")
    cuda = os.path.join(os.path.dirname(os.path.dirname(NVCC)), "include")
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I" + inc,
            "-I" + os.path.join(inc, "torch", "csrc", "api", "include"), "-I" + sysconfig.get_paths()["include"], "-I" + cuda,
            MARSHAL_SRC, "-o", MARSHAL, "-L" + libs, "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda",
            "-Wl,-rpath," + libs]


def _start_marshal():
    """Starts the compilation of _marshal.so; None and the reason where that cannot be."""
    if os.path.exists(MARSHAL):
        os.unlink(MARSHAL)                       # one that no longer fits the library must not stay behind
    try:
        return subprocess.Popen(_marshal_command(), stdout=subprocess.PIPE, stderr=subprocess.STDOUT), None
    except (ImportError, OSError) as e:
        return None, str(e)


def build(force: bool = False, verbose: bool = False) -> str:
    marshal, why = None, None
    if force or _stale(MARSHAL, [MARSHAL_SRC]):
        marshal, why = _start_marshal()
    try:
        if force or _stale(LIB, sources() + glob.glob(os.path.join(CSRC, "*.cuh"))):
            _build_library(verbose)
    finally:
        if marshal:
            out = marshal.communicate()[0].decode()
            if marshal.returncode != 0:
                why = f"exit status {marshal.returncode}\n{out}"
            elif verbose or out.strip():
                sys.stderr.write(out)
        if why:
            sys.stderr.write(f"{MARSHAL_SRC} was not compiled, so the Python binding has no attention operators:\n{why}\n")
    return LIB


def _build_library(verbose):
    objs, procs = [], []
    os.makedirs(OBJ, exist_ok=True)
    for src in sources():
        obj = os.path.join(OBJ, os.path.basename(src)[:-3] + ".o")
        objs.append(obj)
        cmd = [NVCC] + FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-c", src, "-o", obj]
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
    failed = False
    for src, p in procs:
        out = p.communicate()[0].decode()
        if p.returncode != 0:
            failed = True
            sys.stderr.write(f"compiling {src} failed:\n{out}\n")
        elif verbose or out.strip():
            sys.stderr.write(out)
    if failed:
        raise RuntimeError("CUDA build failed")
    subprocess.check_call([NVCC, "-shared", "-o", LIB] + objs + ["-gencode", "arch=compute_100a,code=sm_100a"])


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
