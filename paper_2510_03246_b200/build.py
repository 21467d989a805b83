"""Compile libsp.so (the C-ABI CUDA library) for sm_100a with nvcc, and _binding.so (its native Python binding), in-tree."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "libsp.so")
BINDING = os.path.join(HERE, "_binding.so")
SOURCES = ["sp_api.cu", "sp_gemm_simt.cu", "sp_gemm_tc.cu", "sp_linalg.cu", "sp_linalg_tc.cu", "sp_solve_tc.cu", "sp_elementwise.cu", "sp_mask.cu",
           "sp_profile.cu", "sp_mha.cu", "sp_attention.cu", "sp_attention_tc.cu", "sp_attention_rows.cu", "sp_attention_rows_f32.cu", "sp_linear_few.cu", "sp_loss.cu",
           "sp_norm.cu", "sp_linear_e4m3.cu", "sp_cache.cu", "sp_cache_attention.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr"]


def _nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _binding_command(out: str) -> list:
    import sysconfig

    import torch
    base = os.path.join(os.path.dirname(torch.__file__), "include")
    cuda = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")
    return ["g++", "-O2", "-std=c++17", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
            *(f"-isystem{d}" for d in (base, os.path.join(base, "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"], cuda)),
            "-c", os.path.join(CSRC, "sp_binding.cpp"), "-o", out]


def _stale() -> bool:
    if not os.path.exists(OUT) or not os.path.exists(BINDING):
        return True
    t = min(os.path.getmtime(OUT), os.path.getmtime(BINDING))
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(HERE, "..", "include", "sp.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Build libsp.so if it is missing or older than its sources; returns its path."""
    if not force and not _stale():
        return OUT
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    objs = []
    procs = []
    for src in SOURCES:
        obj = os.path.join(objdir, src.replace(".cu", ".o"))
        cmd = [_nvcc(), *NVCC_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas")
            cmd.insert(2, "-v")
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    binding = os.path.join(objdir, "sp_binding.o")
    procs.append(("sp_binding.cpp", subprocess.Popen(_binding_command(binding), stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = False
    for src, p in procs:
        out, _ = p.communicate()
        if verbose or p.returncode != 0:
            sys.stderr.write(f"--- {src}\n{out}\n")
        failed |= p.returncode != 0
    if failed:
        raise RuntimeError("nvcc failed")
    link = [_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-Xlinker", "-soname=libsp.so", "-o", OUT, *objs]
    subprocess.run(link, check=True)
    import torch
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    subprocess.run(["g++", "-shared", "-o", BINDING, binding, OUT, f"-L{lib}", "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python",
                    "-Wl,-rpath,$ORIGIN", f"-Wl,-rpath,{lib}"], check=True)
    return OUT


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
