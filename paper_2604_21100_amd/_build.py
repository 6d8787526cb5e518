"""Builds libpdn.so (HIP kernels for gfx950 + the C ABI) in-tree with hipcc, and
with the host compiler the part of the binding that is compiled
(_pdn_torch, where torch is there)."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libpdn.so")
TORCH_LIB = os.path.join(HERE, "_pdn_torch.so")
BUILD_DIR = os.path.join(HERE, "_build")

SOURCES = ["pdn_host.cpp", "pdn_fwd.hip", "pdn_bwd.hip", "pdn_scan.hip",
           "pdn_rscan.hip", "pdn_step.hip", "pdn_slots.hip",
           "pdn_slot_chunks.hip", "pdn_slot_runs.hip", "pdn_verify.hip",
           "pdn_block_host.cpp", "pdn_block.hip", "pdn_logits.hip"]

# Packed-fp32 VALU ops are disabled for all device code (they have produced
# silent wrong results on this hardware generation); hipcc's host pass warns
# that it does not know the feature, which is harmless.
HIP_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(ROOT, "include"), "-Wall", "-Wno-unused-result",
]


def _hipcc():
    h = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(h):
        raise RuntimeError("hipcc not found; the HIP library cannot be built")
    return h


def _compile(src, verbose):
    obj = os.path.join(BUILD_DIR, os.path.basename(src) + ".o")
    cmd = [_hipcc(), *HIP_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{r.stdout}\n{r.stderr}")
    return obj


def build_torch(verbose: bool = False):
    """The binding's compiled part, against the torch that is installed (its
    place and ABI asked of an interpreter of its own, so that this one maps no HIP)."""
    ask = ("import torch; from torch.utils.cpp_extension import include_paths, library_paths; "
           "print(int(torch._C._GLIBCXX_USE_CXX11_ABI), *include_paths(), sep='\\n'); print('--', *library_paths(), sep='\\n')")
    r = subprocess.run([sys.executable, "-c", ask], capture_output=True, text=True)
    if r.returncode != 0:
        if "ModuleNotFoundError" in r.stderr:   # no torch: the C ABI alone
            return None
        raise RuntimeError(f"torch does not say where it is:\n{r.stderr}")
    abi, *paths = r.stdout.split("\n")[:-1]
    at = paths.index("--")
    tmp = TORCH_LIB + ".tmp"
    cmd = [shutil.which("g++") or "c++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
           f"-D_GLIBCXX_USE_CXX11_ABI={abi}", "-I" + sysconfig.get_paths()["include"],
           *("-I" + p for p in paths[:at]), os.path.join(CSRC, "pdn_torch.cpp"), "-o", tmp,
           *("-L" + p for p in paths[at + 1:]), "-ltorch_python", "-ltorch_cpu", "-lc10"]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"pdn_torch.cpp failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, TORCH_LIB)
    return TORCH_LIB


def build(verbose: bool = False) -> str:
    """Compile every source for gfx950, link libpdn.so and build _pdn_torch;
    returns libpdn.so's path."""
    os.makedirs(BUILD_DIR, exist_ok=True)
    with ThreadPoolExecutor(max_workers=min(4, len(SOURCES))) as ex:
        objs = list(ex.map(lambda s: _compile(s, verbose), SOURCES))
    tmp = LIB + ".tmp"
    cmd = [_hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", tmp]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    build_torch(verbose)   # (after the library, which does without it)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
