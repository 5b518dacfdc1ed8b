"""Builds libmlpmoe.so (the C-ABI library) for gfx950 with hipcc, in-tree.

hipcc cross-compiles without a GPU.  Usage: python -m paper_2511_21089_amd.build [--force]
"""
from __future__ import annotations

import concurrent.futures
import os
import subprocess
import sys

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG_DIR)
CSRC = os.path.join(PKG_DIR, "csrc")
BUILD_DIR = os.path.join(PKG_DIR, "_build")
LIB_PATH = os.path.join(PKG_DIR, "libmlpmoe.so")

SOURCES = ["mlpmoe_api.cpp", "kernels_generic.hip", "kernels_mfma.hip", "kernels_decode.hip",
           "kernels_fade.hip", "route_api.cpp", "kernels_route.hip", "w4_api.cpp", "kernels_w4.hip", "kernels_w4_tiles.hip"]
HEADERS = [os.path.join(CSRC, "internal.h"), os.path.join(CSRC, "w4_common.h"), os.path.join(ROOT, "include", "mlpmoe.h")]

HIPCC = "/opt/rocm/bin/hipcc"
# packed fp32 VALU instructions are switched off for device code: the compiler would otherwise form them
# from ordinary float arithmetic, and some of their forms have given wrong results on this hardware
COMMON = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fvisibility=hidden",
          "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
          "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-Wall", "-Wno-unused-function"]


def _compile(src: str) -> str:
    obj = os.path.join(BUILD_DIR, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC] + COMMON + ["-x", "hip", "-c", os.path.join(CSRC, src), "-o", obj]
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in res.stdout.splitlines() if "not a recognized feature" not in l)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed for %s:\n%s" % (src, out))
    if out.strip():
        sys.stderr.write(out + "\n")
    return obj


def is_stale() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    t = os.path.getmtime(LIB_PATH)
    deps = [os.path.join(CSRC, s) for s in SOURCES] + HEADERS
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = True, out: str = LIB_PATH) -> str:
    """Compile every translation unit and link the shared library; returns its path."""
    if not force and not is_stale():
        return LIB_PATH
    os.makedirs(BUILD_DIR, exist_ok=True)
    with concurrent.futures.ThreadPoolExecutor(max_workers=4) as ex:
        objs = list(ex.map(_compile, SOURCES))
    tmp = out + ".tmp%d" % os.getpid()
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp] + objs
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if res.returncode != 0:
        raise RuntimeError("link failed:\n" + res.stdout)
    os.replace(tmp, out)
    return out


if __name__ == "__main__":
    print(build(force=True))
