"""Build the C-ABI library ``libdynamo.so`` in-tree with nvcc for sm_100a (no GPU needed to compile).

Every ``.cu`` file is compiled to its own object (in parallel; only the stale ones) and the objects are linked
into the shared library.  No file uses relocatable device code, so plain ``-c`` objects link.  ``torch_binding.cpp`` becomes
an extension module beside it (``_native.so``), built with the host compiler against the installed torch's headers.
"""
from __future__ import annotations

import hashlib
import json
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "build")
LIB = os.path.join(HERE, "libdynamo.so")
SOURCES = ["api.cu", "pack.cu", "route.cu", "switch.cu", "stats.cu", "ffn_stream.cu", "ffn_tc2.cu", "ffn_fold.cu",
           "noalloc.cu", "assign.cu", "downside.cu", "debug.cu", "dispatch.cu", "norm_join.cu", "linear.cu"]
ARCH = ["-gencode", "arch=compute_100a,code=sm_100a"]
CFLAGS = ARCH + ["-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC"]
NATIVE = os.path.join(HERE, "_native.so")
NATIVE_SOURCE = "torch_binding.cpp"
LFLAGS = ARCH + ["-shared", "-Xcompiler", "-fPIC", "-cudart", "static"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    return "nvcc"


def _headers():
    hs = [os.path.join(CSRC, f) for f in sorted(os.listdir(CSRC)) if f.endswith((".cuh", ".h"))]
    hs.append(os.path.join(os.path.dirname(HERE), "include", "dynamo.h"))
    return hs


def _digest(paths) -> str:
    h = hashlib.sha1()
    for p in paths:
        with open(p, "rb") as f:
            h.update(f.read())
    return h.hexdigest()


def _compile(src: str, verbose: bool) -> None:
    obj = os.path.join(OBJ, os.path.splitext(src)[0] + ".o")
    cmd = [_nvcc()] + CFLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-c", "-o", obj, os.path.join(CSRC, src)]
    subprocess.check_call(cmd)


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Staleness goes by content (a digest of every source with all headers, kept beside the objects), not by
    modification times, which a copy of the tree does not preserve."""
    os.makedirs(OBJ, exist_ok=True)
    manifest_path = os.path.join(OBJ, "manifest.json")
    try:
        with open(manifest_path) as f:
            manifest = json.load(f)
    except (OSError, ValueError):
        manifest = {}
    hdr = _digest(_headers())
    want = {s: _digest([os.path.join(CSRC, s)]) + hdr for s in SOURCES}
    stale = [s for s in SOURCES
             if force or manifest.get(s) != want[s] or not os.path.exists(os.path.join(OBJ, os.path.splitext(s)[0] + ".o"))]
    if stale:
        with ThreadPoolExecutor(max_workers=min(len(stale), os.cpu_count() or 4)) as pool:
            list(pool.map(lambda s: _compile(s, verbose), stale))
    objs = [os.path.join(OBJ, os.path.splitext(s)[0] + ".o") for s in SOURCES]
    if stale or not os.path.exists(LIB) or manifest.get("__sources__") != SOURCES:
        subprocess.check_call([_nvcc()] + LFLAGS + ["-o", LIB] + objs)
        want["__sources__"] = SOURCES
        with open(manifest_path, "w") as f:
            json.dump(want, f)
    build_native(force)
    return LIB


def build_native(force: bool = False) -> str:
    """The extension module; built again when its source, the header or the installed torch or Python is another."""
    import sysconfig

    import torch
    from torch.utils import cpp_extension

    manifest_path = os.path.join(OBJ, "native.json")
    want = [_digest([os.path.join(CSRC, NATIVE_SOURCE), _headers()[-1]]), torch.__version__, sys.version]
    try:
        with open(manifest_path) as f:
            have = json.load(f)
    except (OSError, ValueError):
        have = None
    if force or have != want or not os.path.exists(NATIVE):
        cuda = os.path.dirname(os.path.dirname(os.path.realpath(_nvcc()))) if os.path.sep in _nvcc() else "/usr/local/cuda"
        include = cpp_extension.include_paths() + [sysconfig.get_paths()["include"], os.path.join(cuda, "include")]
        torch_lib = os.path.join(os.path.dirname(torch.__file__), "lib")
        cmd = ([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared",
                f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}"] + [f"-isystem{p}" for p in include] +
               ["-o", NATIVE, os.path.join(CSRC, NATIVE_SOURCE), f"-L{HERE}", "-l:libdynamo.so", f"-L{torch_lib}", "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_cuda",
                "-ltorch_python", "-Wl,-rpath,$ORIGIN"])
        subprocess.check_call(cmd)
        with open(manifest_path, "w") as f:
            json.dump(want, f)
    return NATIVE


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv))
