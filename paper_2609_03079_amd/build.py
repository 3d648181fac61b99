"""Compile the gfx950 HIP library ``liblsffn.so`` in-tree with hipcc, and the Python module that
marshals the operators' arguments (``_lsops``) with g++."""
from __future__ import annotations

import concurrent.futures as cf
import hashlib
import os
import subprocess
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "liblsffn.so")
BINDING = os.path.join(HERE, "_lsops" + sysconfig.get_config_var("EXT_SUFFIX"))
SOURCES = ["ls_api.hip", "ls_kernels.hip", "ls_decode.hip", "ls_mfma.hip", "ls_hash.hip", "ls_stage.hip",
           "ls_ops_api.hip", "ls_rows.hip", "ls_linear.hip", "ls_attend.hip"]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # no packed-fp32 instructions in any generated code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


ROOT = os.path.dirname(HERE)


def source_digest() -> str:
    """sha256 over the library's sources (every file in csrc/, the public headers and this
    build script), each as its path relative to the repository and its bytes, in path order."""
    files = [os.path.join(CSRC, f) for f in os.listdir(CSRC)
             if f.endswith((".hip", ".h", ".cpp"))]
    files += [os.path.join(ROOT, "include", h) for h in ("ls_ffn.h", "ls_ops.h")] + [os.path.abspath(__file__)]
    h = hashlib.sha256()
    for path in sorted(files, key=lambda p: os.path.relpath(p, ROOT)):
        h.update(os.path.relpath(path, ROOT).encode() + b"\0")
        with open(path, "rb") as fh:
            h.update(fh.read())
        h.update(b"\0")
    return h.hexdigest()


def _rocm() -> str:
    return os.environ.get("ROCM_PATH", "/opt/rocm")


def _hipcc() -> str:
    p = os.path.join(_rocm(), "bin", "hipcc")
    return p if os.path.exists(p) else "hipcc"


def _build_binding(digest: str) -> None:
    """Compile ls_binding.cpp against torch and the library beside it."""
    import torch
    from torch.utils.cpp_extension import include_paths, library_paths
    inc = [f"-I{d}" for d in [*include_paths(), sysconfig.get_paths()["include"], os.path.join(_rocm(), "include")]]
    lib = [f"-L{d}" for d in library_paths()]
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-Wall", "-D__HIP_PLATFORM_AMD__=1",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f'-DLS_BUILD_DIGEST="{digest}"', *inc,
           os.path.join(CSRC, "ls_binding.cpp"), "-o", BINDING + ".tmp", LIB, *lib, "-ltorch_python", "-ltorch_cpu", "-lc10",
           "-Wl,-rpath,$ORIGIN"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed for ls_binding.cpp:\n{r.stderr}")
    os.replace(BINDING + ".tmp", BINDING)


def build(verbose: bool = False) -> str:
    """Compile every source to an object, link the shared library and the Python module, return
    the library's path."""
    os.makedirs(BUILD, exist_ok=True)
    srcs = [s for s in SOURCES if os.path.exists(os.path.join(CSRC, s))]

    digest = source_digest()

    def compile_one(src: str) -> str:
        obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
        cmd = [_hipcc(), *HIPCC_FLAGS, f'-DLS_BUILD_DIGEST="{digest}"', "-c", os.path.join(CSRC, src),
               "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"hipcc failed for {src}:\n{r.stderr}")
        if verbose and r.stderr:
            print(r.stderr)
        return obj

    with cf.ThreadPoolExecutor(max_workers=len(srcs)) as ex:
        objs = list(ex.map(compile_one, srcs))
    tmp = LIB + ".tmp"
    cmd = [_hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", "-Wl,-soname,liblsffn.so", "-o", tmp, *objs, "-lpthread"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, LIB)
    _build_binding(digest)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
