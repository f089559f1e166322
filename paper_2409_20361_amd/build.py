"""Build librrs.so (the C-ABI HIP library) in-tree for gfx950 with hipcc, and _torch_calls.so
(the calls on torch tensors) with the host compiler.

Each source is compiled to an object in parallel, then linked into
paper_2409_20361_amd/librrs.so and _torch_calls.so. Always recompiles.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "librrs.so")
TORCH_LIB = os.path.join(PKG, "_torch_calls.so")
OBJDIR = os.path.join(PKG, "_build")

SOURCES = ["rrs_api.cpp", "rrs_gemm_route.cpp", "rrs_quant.hip", "rrs_weight.hip", "rrs_gemm.hip",
           "rrs_gemm_small.hip", "rrs_gemm_decode.hip", "rrs_quant_wave.hip", "rrs_reorder.hip", "rrs_quant_rows.hip",
           "rrs_gemm_stream.hip", "rrs_gemm_stream_gather.hip", "rrs_gemm_mid.hip",
           "rrs_gemm_fp6.hip", "rrs_noalloc.hip", "rrs_kv_api.cpp", "rrs_kv_append.hip",
           "rrs_attention.hip", "rrs_evict.hip"]

# Per-source code-generation options on top of COMMON.
# rrs_gemm_stream_gather.hip: keep MFMA results in VGPRs (the per-block
#   rescale reads every accumulator; in AGPRs each read is an extra copy).
# rrs_gemm_fp6.hip: the same (every partial is read by the rescale).
# rrs_attention.hip: the same (logits are read by the softmax, sums rescaled).
EXTRA = {"rrs_gemm_stream_gather.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
         "rrs_gemm_fp6.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
         "rrs_attention.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"]}

# -packed-fp32-ops: no v_pk_{add,mul,fma}_f32 in any kernel.
# -ffp-contract=off: every rounding in the rotation and scale chain is an
#   explicit single IEEE operation; the GEMM epilogue asks for fma explicitly.
COMMON = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-ffp-contract=off", "-fno-fast-math",
    "-Wall", "-Wno-unused-function", "-Wno-unknown-warning-option",
    "-I" + INCLUDE, "-I" + CSRC,
]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found (ROCm is required to build librrs.so)")


def _run(cmd, what: str) -> str:
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{what} failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    return r.stderr


def _compile_torch() -> str:
    """rrs_torch.cpp: host code only, against the headers of the torch that is installed."""
    import torch
    root = os.path.dirname(torch.__file__)
    obj = os.path.join(OBJDIR, "rrs_torch.o")
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-Wall",
           "-D__HIP_PLATFORM_AMD__", "-DUSE_ROCM",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I" + INCLUDE]
    for inc in (os.path.join(root, "include"),
                os.path.join(root, "include", "torch", "csrc", "api", "include"),
                sysconfig.get_paths()["include"],
                os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include")):
        cmd += ["-isystem", inc]
    noise = _run(cmd + ["-c", os.path.join(CSRC, "rrs_torch.cpp"), "-o", obj], "compile")
    if noise:
        sys.stderr.write(f"[build] rrs_torch.cpp:\n{noise}\n")
    return obj


def _link_torch(obj: str) -> None:
    import torch
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    tmp = TORCH_LIB + ".tmp"
    _run([os.environ.get("CXX", "g++"), "-shared", "-o", tmp, obj, "-L" + PKG, "-l:librrs.so",
          "-L" + libs, "-lc10", "-lc10_hip", "-ltorch_cpu", "-ltorch_python",
          "-Wl,-rpath,$ORIGIN:" + libs], "link")
    os.replace(tmp, TORCH_LIB)


def _compile(src: str) -> str:
    obj = os.path.join(OBJDIR, os.path.splitext(src)[0] + ".o")
    lang = ["-x", "hip"] if src.endswith(".hip") else []
    cmd = [hipcc()] + COMMON + EXTRA.get(src, []) + ["-c"] + lang + [os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    # hipcc's host pass does not know the packed-fp32 feature; that warning is expected.
    noise = [ln for ln in r.stderr.splitlines()
             if ln.strip() and "packed-fp32-ops" not in ln and "not a recognized feature" not in ln]
    if noise:
        sys.stderr.write(f"[build] {src}:\n" + "\n".join(noise) + "\n")
    return obj


def build(verbose: bool = False) -> str:
    os.makedirs(OBJDIR, exist_ok=True)
    with ThreadPoolExecutor(max_workers=min(len(SOURCES) + 1, os.cpu_count() or 4)) as ex:
        torch_obj = ex.submit(_compile_torch)
        objs = list(ex.map(_compile, SOURCES))
        torch_obj = torch_obj.result()
    tmp = LIB + ".tmp"
    cmd = [hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    _link_torch(torch_obj)
    if verbose:
        print(f"[build] wrote {LIB} and {TORCH_LIB}")
    return LIB


if __name__ == "__main__":
    build(verbose=True)
