"""Builds the CUDA library in-tree: ``python -m paper_2607_16184_b200.build``."""
from __future__ import annotations

import glob
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libpw.so")
MODULE = os.path.join(HERE, "_pwtorch.so")         # argument marshalling for torch tensors
MODULE_SOURCE = os.path.join(CSRC, "pw_torch.cpp")

NVCC_FLAGS = ["-std=c++17", "-O3", "-lineinfo", "-gencode", "arch=compute_100a,code=sm_100a", "-Xcompiler", "-fPIC",
              "-shared", "-cudart", "static"]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def needs_build() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + [os.path.join(HERE, "..", "include", "pw.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def module_stamp() -> str:
    """What the module has to be built for to load: it uses torch's C++ interface and this Python's."""
    import torch
    return "torch %s, python %d.%d" % ((torch.__version__,) + sys.version_info[:2])


def module_is_current() -> bool:
    deps = (MODULE_SOURCE, os.path.join(HERE, "..", "include", "pw.h"))
    if not os.path.exists(MODULE) or any(os.path.getmtime(d) > os.path.getmtime(MODULE) for d in deps):
        return False
    with open(MODULE, "rb") as f:
        return (module_stamp() + "\0").encode() in f.read()


def build_module(force: bool = False) -> str:
    """The CPython module that marshals torch tensors for the calls of libpw.so."""
    if not force and module_is_current():
        return MODULE
    import torch
    from torch.utils import cpp_extension
    dirs = cpp_extension.include_paths() + [sysconfig.get_paths()["include"], os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")]
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-fPIC", "-shared", "-Wall", "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch.compiled_with_cxx11_abi()),
                           '-DPW_BUILT_FOR="%s"' % module_stamp()] + [a for d in dirs for a in ("-isystem", d)] +
                          [MODULE_SOURCE, "-o", MODULE, "-L" + libs, "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python", "-L" + HERE, "-l:libpw.so",
                           "-Wl,-rpath,$ORIGIN"])
    return MODULE


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not needs_build():
        build_module()
        return LIB
    objs = []
    procs = []
    for src in sources():
        obj = src[:-3] + ".o"
        cmd = ["nvcc"] + [f for f in NVCC_FLAGS if f != "-shared"] + (["-Xptxas", "-v"] if verbose else []) + \
              ["-c", src, "-o", obj]
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    failed = False
    for src, p in procs:
        out, _ = p.communicate()
        if verbose or p.returncode != 0:
            sys.stderr.write(out)
        failed |= p.returncode != 0
    if failed:
        raise RuntimeError("nvcc failed")
    subprocess.check_call(["nvcc", "-shared", "-cudart", "static", "-gencode", "arch=compute_100a,code=sm_100a",
                           "-o", LIB] + objs)
    build_module(force)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
