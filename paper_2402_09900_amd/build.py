"""Build libmemoroid.so (hand-written HIP for gfx950) in-tree with hipcc, and
_torch_layer.so (calls on torch tensors and autograd nodes, host code) with g++.

    python -m paper_2402_09900_amd.build

Both are always rebuilt (a few minutes); the results land next to this file,
where the binding loads them from.  Without torch the library alone is built.
"""
from __future__ import annotations

import glob
import importlib.util
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libmemoroid.so")
LAYER = os.path.join(HERE, "_torch_layer.so")
ARCH = "gfx950"

FLAGS = [
    "-O3", "-std=c++17", "-fPIC", "-shared", "--offload-arch=" + ARCH,
    # no packed-fp32 instructions anywhere in the device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # every atomic here is issued by one lane; the compiler's wave-wide
    # atomic rewrite would read the result back at once, stalling the tile's
    # loads behind the atomic's round trip
    "-mllvm", "-amdgpu-atomic-optimizer-strategy=None",
    "-Wall", "-Wno-unused-command-line-argument",
    "-I", os.path.join(ROOT, "include"),
]


def sources():
    return sorted(glob.glob(os.path.join(HERE, "csrc", "*.hip")))


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    return subprocess.Popen(cmd)


def _done(process):
    if process.wait():
        raise subprocess.CalledProcessError(process.returncode, process.args)


def _layer_commands(obj, tmp):
    """The torch layer's compile and link; it calls the library, which is found beside it."""
    from torch.utils import cpp_extension

    includes = cpp_extension.include_paths("cuda") + [sysconfig.get_paths()["include"]]
    return (["g++", "-O2", "-std=c++17", "-fPIC", "-Wall", "-Wno-unknown-pragmas", "-D__HIP_PLATFORM_AMD__=1",
             "-DUSE_ROCM=1", "-DTORCH_EXTENSION_NAME=_torch_layer", "-I", os.path.join(ROOT, "include")]
            + [a for d in includes for a in ("-isystem", d)]
            + ["-c", os.path.join(HERE, "csrc", "torch_layer.cpp"), "-o", obj],
            ["g++", "-shared", obj, "-o", tmp, "-L", HERE, "-lmemoroid", "-Wl,-rpath,$ORIGIN"]
            + [a for d in cpp_extension.library_paths("cuda") for a in ("-L", d)]
            + ["-lc10", "-lc10_hip", "-ltorch_cpu", "-ltorch_hip", "-ltorch", "-ltorch_python"])


def build(verbose: bool = False) -> str:
    end = ".tmp%d" % os.getpid()
    obj = os.path.join(HERE, "torch_layer%s.o" % end)
    layer = None
    if importlib.util.find_spec("torch") is not None:
        compile_layer, link_layer = _layer_commands(obj, LAYER + end)
        layer = _run(compile_layer, verbose)
    else:
        print("no torch here: building libmemoroid.so alone", flush=True)
    library = _run(["hipcc"] + FLAGS + ["-o", LIB + end] + sources(), verbose)
    try:
        _done(library)
        os.replace(LIB + end, LIB)
        if layer is not None:
            _done(layer)
            _done(_run(link_layer, verbose))
            os.replace(LAYER + end, LAYER)
    finally:
        if layer is not None:
            layer.wait()
        if os.path.exists(obj):
            os.remove(obj)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
