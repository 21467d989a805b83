"""Compile libsp.so (the C-ABI CUDA library) for sm_100a with nvcc, and _binding.so (its native Python binding), in-tree."""
from __future__ import annotations

import os
import subprocess
import sys
import warnings

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


def _binding_link(obj: str) -> list:
    import torch
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    return ["g++", "-shared", "-o", BINDING, obj, OUT, f"-L{lib}", "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python", "-Wl,-rpath,$ORIGIN",
            f"-Wl,-rpath,{lib}"]


def _older(path: str, sources) -> bool:
    return not os.path.exists(path) or any(os.path.getmtime(s) > os.path.getmtime(path) for s in sources)


def _stale() -> tuple[bool, bool]:
    """Whether libsp.so and _binding.so are missing or older than what they are made of."""
    header, binding = os.path.join(HERE, "..", "include", "sp.h"), os.path.join(CSRC, "sp_binding.cpp")
    library = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f != "sp_binding.cpp"]
    return _older(OUT, [header, *library]), _older(BINDING, [header, binding])


def build(force: bool = False, verbose: bool = False) -> str:
    """Build libsp.so, and _binding.so, if they are missing or older than their sources; returns the library's path.  Without Python's or torch's
    headers there is no _binding.so: a warning says so, and the calls that need it raise (api._binding); all others need libsp.so alone."""
    library, binding = (True, True) if force else _stale()
    if not library and not binding:
        return OUT
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    objs = []
    procs = []
    for src in SOURCES if library else ():
        obj = os.path.join(objdir, src.replace(".cu", ".o"))
        cmd = [_nvcc(), *NVCC_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas")
            cmd.insert(2, "-v")
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    obj = os.path.join(objdir, "sp_binding.o")
    compiled, log = None, ""
    if binding:
        try:
            compiled = subprocess.Popen(_binding_command(obj), stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        except (OSError, ImportError) as e:          # (no compiler, no torch)
            log = str(e)
    failed = False
    for src, p in procs:
        out, _ = p.communicate()
        if verbose or p.returncode != 0:
            sys.stderr.write(f"--- {src}\n{out}\n")
        failed |= p.returncode != 0
    if compiled:
        log, _ = compiled.communicate()
    if failed:
        raise RuntimeError("nvcc failed")
    if library:
        link = [_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-Xlinker", "-soname=libsp.so", "-o", OUT, *objs]
        subprocess.run(link, check=True)
    if binding:
        linked = compiled is not None and compiled.returncode == 0 and subprocess.run(_binding_link(obj)).returncode == 0
        if verbose or not linked:
            sys.stderr.write(f"--- sp_binding.cpp\n{log}\n")
        if not linked:
            if os.path.exists(BINDING):
                os.remove(BINDING)                   # (of another header or source)
            warnings.warn("_binding.so could not be built: sp_rms_norm, sp_linear_e4m3, sp_cache_* and what calls them will raise")
    return OUT


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
