"""Builds libspecverify.so (HIP, gfx950) in-tree with hipcc, and _native.so, the marshalling of tensors for its shortest
calls, with the host compiler.  The library needs neither that compiler nor the headers of torch and Python."""
from __future__ import annotations

import os
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libspecverify.so")
NATIVE = os.path.join(HERE, "_native.so")
SOURCES = ["attention.hip", "attention_reuse.hip", "spec_verify.hip", "forward.hip", "sampler.hip", "gemm.hip",
           "elementwise.hip", "probe.hip", "decode.hip", "lookahead.hip", "q8_rows.hip", "q8_gemm.hip", "kv8.hip",
           "filter_sample.hip", "prompt_rows.hip", "prompt_gemm.hip", "prompt_attention.hip"]
# packed-fp32 instructions are disabled for all device code.  The first kernel arguments (up to 14 dwords, whole structs
# excepted) come in scalar registers with the wavefront instead of by a load that every wavefront waits for before its
# first address: a step is a chain of small launches (1B shape, batch 1, 120 of them: 812 -> 787 us).  Kernels list
# what their first loads need in front.
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-mllvm", "-amdgpu-kernarg-preload-count=16",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
# Per-source additions.  The attention kernels: matrix instructions take their accumulators in ordinary vector
# registers; left to its default the compiler parks them in the accumulation registers and copies all
# 32 of them out and back around every block's products (the rare rescaling is vector arithmetic).
# The GEMM kernels keep the default: several of their variants measured slower with this option.
SOURCE_FLAGS = {"attention.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
                "attention_reuse.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
                "kv8.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
                "prompt_attention.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"]}
OBJ_DIR = os.path.join(HERE, "_build")


def _hipcc() -> str:
    for c in (shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("hipcc not found: cannot build libspecverify.so")


def _native_command() -> list:
    import sysconfig

    import torch
    base = os.path.dirname(torch.__file__)
    cxx = shutil.which("g++") or shutil.which("c++")
    if not cxx:
        raise RuntimeError("no host compiler found: cannot build _native.so")
    return [cxx, "-std=c++17", "-O2", "-shared", "-fPIC", "-DUSE_ROCM", "-D__HIP_PLATFORM_AMD__=1",
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f"-I{base}/include",
            f"-I{base}/include/torch/csrc/api/include", f"-I{sysconfig.get_paths()['include']}", "-o", NATIVE,
            os.path.join(CSRC, "native.cpp"), f"-L{base}/lib", "-ltorch_python", "-ltorch_cpu", "-lc10"]


def sources_newer_than_lib(built: str = LIB) -> bool:
    if not os.path.exists(built):
        return True
    t = os.path.getmtime(built)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + \
           [os.path.join(HERE, "..", "include", f) for f in os.listdir(os.path.join(HERE, "..", "include"))]
    return any(os.path.getmtime(d) > t for d in deps)


def _report(r, verbose: bool) -> None:
    noise = "packed-fp32-ops"
    if verbose or r.returncode:
        print("\n".join(l for l in (r.stdout + r.stderr).splitlines() if noise not in l and l.strip()))


def build_library(force: bool = False, verbose: bool = False) -> str:
    if not force and not sources_newer_than_lib(LIB):
        return LIB
    os.makedirs(OBJ_DIR, exist_ok=True)
    hipcc = _hipcc()

    def compile_one(src):
        obj = os.path.join(OBJ_DIR, src.replace(".hip", ".o"))
        cmd = [hipcc] + FLAGS + SOURCE_FLAGS.get(src, []) + ["-c", "-o", obj, os.path.join(CSRC, src)]
        return obj, subprocess.run(cmd, capture_output=True, text=True)

    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as pool:   # one hipcc process per source
        done = list(pool.map(compile_one, SOURCES))
    for _, r in done:
        _report(r, verbose)
    if any(r.returncode for _, r in done):
        raise RuntimeError("hipcc failed building libspecverify.so")
    r = subprocess.run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + [o for o, _ in done],
                       capture_output=True, text=True)
    _report(r, verbose)
    if r.returncode:
        raise RuntimeError("hipcc failed linking libspecverify.so")
    return LIB


def build_native(force: bool = False, verbose: bool = False) -> str:
    if not force and not sources_newer_than_lib(NATIVE):
        return NATIVE
    r = subprocess.run(_native_command(), capture_output=True, text=True)
    _report(r, verbose)
    if r.returncode:
        raise RuntimeError("the host compiler failed building _native.so")
    return NATIVE


if __name__ == "__main__":
    print(build_library(force=True, verbose=True))
    print(build_native(force=True, verbose=True))
