"""Build libmra.so, libmra_exact.so and libmra_layer.so (the HIP kernels and their C
ABIs, gfx950) and _binding.so, _binding_exact.so and _binding_layer.so (the torch
bindings of ops.py's calls, host code) in-tree.

    python -m paper_2207_10284_amd.build

Sources compile in parallel into <repo>/_build/, then link into
paper_2207_10284_amd/.
"""
from __future__ import annotations

import concurrent.futures as cf
import importlib.util
import os
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "libmra.so")
LIB_EXACT = os.path.join(PKG, "libmra_exact.so")
LIB_LAYER = os.path.join(PKG, "libmra_layer.so")
BINDING = os.path.join(PKG, "_binding.so")
BINDING_EXACT = os.path.join(PKG, "_binding_exact.so")
BINDING_LAYER = os.path.join(PKG, "_binding_layer.so")
SOURCES = ["api.cpp", "pool.hip", "coarse.hip", "select.hip", "select_global.hip", "tile.hip",
           "bwd.hip", "multilevel.hip", "noalloc.hip"]
EXACT_SOURCES = ["exact_api.cpp", "exact_fwd.hip", "exact_bwd.hip"]
LAYER_SOURCES = ["layer_api.cpp", "rotary.hip", "fp4_cache.hip", "fp4_attention.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"
FLAGS = [
    "-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}",
    # packed fp32 VALU ops stay off: hipcc would otherwise form them from
    # ordinary float code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # matrix-core results stay in ordinary VGPRs, so the rare rescale of the
    # accumulators needs no AGPR round trips
    "-mllvm", "-amdgpu-mfma-vgpr-form=1",
    "-I", INCLUDE, "-I", CSRC,
]


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    return obj


def _build_binding(source: str, binding: str) -> str:
    """A torch binding: host code against the installed torch's headers; it
    takes its library's entry points by address, so it does not link to it."""
    torch = os.path.dirname(importlib.util.find_spec("torch").origin)
    inc = [os.path.join(torch, "include"), os.path.join(torch, "include", "torch", "csrc", "api", "include"),
           "/opt/rocm/include", sysconfig.get_paths()["include"]]
    tmp = binding + ".tmp"
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-D__HIP_PLATFORM_AMD__=1",
           "-DUSE_ROCM", "-I", INCLUDE, *(f for d in inc for f in ("-isystem", d)), os.path.join(CSRC, source),
           "-L", os.path.join(torch, "lib"), "-lc10", "-lc10_hip", "-ltorch_cpu", "-ltorch", "-ltorch_python",
           "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, binding)
    return binding


def _link(objs, lib: str) -> None:
    tmp = lib + ".tmp"
    cmd = [HIPCC, "-shared", "-fPIC", f"--offload-arch={ARCH}", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, lib)


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=8) as ex:
        bindings = [ex.submit(_build_binding, "binding.cpp", BINDING),
                    ex.submit(_build_binding, "exact_binding.cpp", BINDING_EXACT),
                    ex.submit(_build_binding, "layer_binding.cpp", BINDING_LAYER)]
        exact = [ex.submit(_compile, s) for s in EXACT_SOURCES]
        layer = [ex.submit(_compile, s) for s in LAYER_SOURCES]
        objs = list(ex.map(_compile, SOURCES))
        exact = [f.result() for f in exact]
        layer = [f.result() for f in layer]
        for b in bindings:
            b.result()
    _link(objs, LIB)
    _link(exact, LIB_EXACT)
    _link(layer, LIB_LAYER)
    if verbose:
        print(f"built {LIB}, {LIB_EXACT}, {LIB_LAYER}, {BINDING}, {BINDING_EXACT} and {BINDING_LAYER}")
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
