"""Builds the CUDA library in-tree: ``python -m paper_2103_07454_b200.build`` (``--debug``: the
bounds-checked build, ``libeventgrad_debug.so``)."""
from __future__ import annotations

import importlib.util
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
SRC = [os.path.join(HERE, "csrc", "eventgrad.cu"), os.path.join(HERE, "csrc", "eg_norms_static.cu")]
#: the operators around the step: their products may be contracted into fused multiply-adds
OPS = [os.path.join(HERE, "csrc", f) for f in ("eg_residual_norm.cu", "eg_feed_forward.cu")]
LIB = os.path.join(HERE, "libeventgrad.so")
#: torch tensors to C arguments, for the operators
MARSHAL_SRC = os.path.join(HERE, "csrc", "marshal.cpp")
MARSHAL = os.path.join(HERE, "_marshal.so")
#: what it was built for: it fits one interpreter and one torch
MARSHAL_STAMP = os.path.join(HERE, "_build", "_marshal.txt")
LIB_DEBUG = os.path.join(HERE, "libeventgrad_debug.so")
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")

FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
         "-Xcompiler", "-fPIC", "-DEG_FUSED_VPT=1"]
STEP_FLAGS = ["--fmad=false"]  # every fused multiply-add of the step is written out


def sources():
    d = os.path.join(HERE, "csrc")
    return [os.path.join(d, f) for f in sorted(os.listdir(d))] + [
        os.path.join(HERE, "..", "include", "eventgrad.h")]


def _compile(lib: str, extra, force: bool, verbose: bool) -> str:
    newest = max(os.path.getmtime(p) for p in sources())
    if force or not os.path.exists(lib) or os.path.getmtime(lib) < newest:
        flags = FLAGS + list(extra) + (["-Xptxas", "-v"] if verbose else [])
        objects, running = [], []
        os.makedirs(os.path.join(HERE, "_build"), exist_ok=True)
        for src in SRC + OPS:
            obj = os.path.join(HERE, "_build", os.path.basename(lib) + "." + os.path.basename(src) + ".o")
            objects.append(obj)
            running.append(subprocess.Popen([NVCC] + flags + (STEP_FLAGS if src in SRC else []) + ["-c", "-o", obj, src]))
        failed = [p.args for p in running if p.wait() != 0]
        if failed:
            raise subprocess.CalledProcessError(1, failed[0])
        subprocess.run([NVCC] + FLAGS[:2] + ["-shared", "-o", lib] + objects + ["-ldl"], check=True)
    return lib


def _stamp() -> str:
    """Interpreter and torch by version and place, from the latter's files (importing it takes seconds)."""
    top = os.path.dirname(importlib.util.find_spec("torch").origin)
    with open(os.path.join(top, "version.py")) as f:
        return f"{sys.version}\n{sysconfig.get_config_var('SOABI')}\n{top}\n{f.read()}"


def build_marshal(force: bool = False) -> str:
    newest = max(os.path.getmtime(p) for p in (MARSHAL_SRC, os.path.join(HERE, "..", "include", "eventgrad.h")))
    stamp, built_for = _stamp(), None
    if os.path.exists(MARSHAL_STAMP):
        with open(MARSHAL_STAMP) as f:
            built_for = f.read()
    if force or not os.path.exists(MARSHAL) or os.path.getmtime(MARSHAL) < newest or built_for != stamp:
        import torch
        top = os.path.dirname(torch.__file__)
        include = [os.path.join(top, "include"), os.path.join(top, "include", "torch", "csrc", "api", "include"),
                   sysconfig.get_paths()["include"], os.path.join(os.path.dirname(os.path.dirname(NVCC)), "include")]
        subprocess.run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC",
                        f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}"]
                       + [a for d in include for a in ("-isystem", d)] + ["-o", MARSHAL, MARSHAL_SRC, "-L" + os.path.join(top, "lib")]
                       + ["-l" + n for n in ("torch_python", "torch_cuda", "c10_cuda", "torch_cpu", "c10")], check=True)
        os.makedirs(os.path.dirname(MARSHAL_STAMP), exist_ok=True)
        with open(MARSHAL_STAMP, "w") as f:
            f.write(stamp)
    return MARSHAL


def build(force: bool = False, verbose: bool = False) -> str:
    lib = _compile(LIB, [], force, verbose)     # first: the step does without the rest
    build_marshal(force)
    return lib


def build_debug(force: bool = False, verbose: bool = False) -> str:
    """The bounds-checked build (-DEG_DEBUG): every index a kernel forms into a table is compared
    with the table's size first; a miss sets a bit of the context's error word instead of
    touching memory.  Load it with EG_LIBRARY=<path> in the environment."""
    return _compile(LIB_DEBUG, ["-DEG_DEBUG"], force, verbose)


if __name__ == "__main__":
    if "--debug" in sys.argv:
        print(build_debug(force="--force" in sys.argv, verbose="-v" in sys.argv))
    else:
        print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
