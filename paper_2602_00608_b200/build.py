"""Builds libvd.so (the CUDA library behind include/vd.h) in-tree with nvcc for sm_100a, and _vd_torch.so, which hands torch tensors
to its block operators without Python in between."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OBJ = os.path.join(PKG, "build")
LIB = os.path.join(PKG, "libvd.so")
TORCH_LIB = os.path.join(PKG, "_vd_torch.so")
SOURCES = ["vd_api.cu", "kernels_simt.cu", "conv_tc.cu", "conv_split.cu", "conv_f32.cu", "conv_f32_tc.cu", "attn_tc.cu", "wait_probe.cu",
           "block_api.cu", "xattn_plain.cu", "xattn_rows.cu", "xattn_tc.cu", "xattn_f32.cu", "rotary.cu", "gate_norm.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC,-fvisibility=hidden", "-DVD_BUILD",
              "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _newer(target: str, deps) -> bool:
    if not os.path.exists(target):
        return False
    t = os.path.getmtime(target)
    return all(os.path.getmtime(d) <= t for d in deps)


def build(verbose: bool = False, force: bool = False) -> str:
    os.makedirs(OBJ, exist_ok=True)
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))]
    headers += [os.path.join(ROOT, "include", f) for f in ("vd.h", "vd_ops.h", "vd_block.h")]
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")

    def compile_one(src: str) -> str:
        s = os.path.join(CSRC, src)
        o = os.path.join(OBJ, src.replace(".cu", ".o"))
        if force or not _newer(o, [s] + headers):
            cmd = [nvcc, *NVCC_FLAGS, "-c", s, "-o", o]
            if verbose:
                cmd.insert(1, "-Xptxas")
                cmd.insert(2, "-v")
            r = subprocess.run(cmd, capture_output=True, text=True)
            if verbose or r.returncode != 0:
                sys.stderr.write(r.stdout + r.stderr)
            if r.returncode != 0:
                raise RuntimeError(f"nvcc failed for {src}")
        return o

    with ThreadPoolExecutor(max_workers=4) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    if force or not _newer(LIB, objs):
        tmp = LIB + f".tmp{os.getpid()}"
        subprocess.run([nvcc, "-shared", "-o", tmp, *objs, "-lcudart"], check=True)
        os.replace(tmp, LIB)
    try:
        build_torch(verbose, force)
    except (ImportError, OSError, RuntimeError) as e:            # no torch, no g++, other headers: the library does without it
        if os.path.exists(TORCH_LIB):
            os.remove(TORCH_LIB)                                 # (built from an earlier vd_block.h)
        sys.stderr.write(f"_vd_torch.so was not built ({e}): calls of the block operators take the way through ctypes\n")
    return LIB


def build_torch(verbose: bool = False, force: bool = False) -> str:
    import sysconfig

    import torch
    src = os.path.join(CSRC, "vd_torch.cpp")
    headers = [os.path.join(ROOT, "include", f) for f in ("vd.h", "vd_block.h")]
    home = os.path.dirname(torch.__file__)
    if force or not _newer(TORCH_LIB, [src, *headers, os.path.join(home, "version.py")]):
        cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
        tmp = TORCH_LIB + f".tmp{os.getpid()}"
        cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
               "-I", os.path.join(ROOT, "include"), "-I", sysconfig.get_paths()["include"], "-I", os.path.join(home, "include"),
               "-I", os.path.join(home, "include", "torch", "csrc", "api", "include"), "-I", os.path.join(cuda, "include"), src, "-o", tmp,
               "-L", os.path.join(home, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if verbose or r.returncode != 0:
            sys.stderr.write(r.stdout + r.stderr)
        if r.returncode != 0:
            raise RuntimeError("g++ failed for vd_torch.cpp")
        os.replace(tmp, TORCH_LIB)
    return TORCH_LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv, force="-f" in sys.argv))
