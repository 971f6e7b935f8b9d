"""Builds libuniep_moe.so (HIP, gfx950 only) in-tree with hipcc, and the binding's extension module with g++.

Objects and compiler temporaries go to <repo>/_build/; the shared library is
written next to this file so that it travels with the source tree.
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor
from pathlib import Path

PKG = Path(__file__).resolve().parent
CSRC = PKG / "csrc"
LIB = PKG / "libuniep_moe.so"
CALL = PKG / "_call.so"                  # host side of the short calls (csrc/call.cpp)
BUILD = PKG.parent / "_build"
SOURCES = ["route.hip", "forward.hip", "backward.hip", "adapter.hip", "balance.hip", "move.hip", "saved.hip", "mx.hip", "mx_product.hip", "api.hip", "perf_model.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # packed-fp32 VALU forms are kept out of the generated code on purpose
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
]


def _compile(src: str, save_temps: bool) -> Path:
    obj = BUILD / (src + ".o")
    cmd = [HIPCC, *FLAGS, "-c", str(CSRC / src), "-o", str(obj)]
    if save_temps:
        cmd.append("-save-temps=obj")
    r = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{err}")
    if err.strip():
        print(err, file=sys.stderr)
    return obj


def _build_call() -> None:
    """The extension module that checks, allocates and calls for binding.py (host code: g++)."""
    import sysconfig

    import torch
    from torch.utils import cpp_extension
    inc = [f"-I{d}" for d in (*cpp_extension.include_paths(), sysconfig.get_paths()["include"])]
    lib = [f"-L{d}" for d in cpp_extension.library_paths()]
    subprocess.run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                    *inc, str(CSRC / "call.cpp"), "-o", str(CALL), *lib, "-lc10", "-ltorch_cpu", "-ltorch", "-ltorch_python"], check=True)


def build(save_temps: bool = False, jobs: int = 6) -> Path:
    BUILD.mkdir(exist_ok=True)
    with ThreadPoolExecutor(max_workers=jobs) as ex:
        call = ex.submit(_build_call)
        objs = list(ex.map(lambda s: _compile(s, save_temps), SOURCES))
        call.result()
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *map(str, objs), "-o", str(LIB)]
    subprocess.run(cmd, check=True)
    return LIB


if __name__ == "__main__":
    print(build(save_temps="--save-temps" in sys.argv))
