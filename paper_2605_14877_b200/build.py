"""Builds libheatkv.so (CUDA kernels + C ABI) in-tree for sm_100a with nvcc, and the CPython modules beside it: the call sequencer _native and
the paged cache's calls, _paged."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libheatkv.so")
NATIVE = os.path.join(HERE, "_native" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))
PAGED = os.path.join(HERE, os.path.basename(NATIVE).replace("_native", "_paged"))
SOURCES = ["schedule.cpp", "plan.cpp", "split.cpp", "api.cu", "attn_generic.cu", "attn_tc.cu", "attn_pair.cu", "calib_tc.cu", "cache_kernels.cu",
           "paged_api.cu", "paged_tables.cu", "paged_select.cu", "paged_small.cu", "paged_tc.cu",
           "paged_rows.cu", "paged4_rows.cu", "paged4_small.cu"]


def _stale() -> bool:
    built = (LIB, NATIVE, PAGED)
    if not all(os.path.exists(p) for p in built):
        return True
    lib_t = min(os.path.getmtime(p) for p in built)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", "heatkv.h")]
    return any(os.path.getmtime(p) > lib_t for p in deps)


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compiles every translation unit for sm_100a and links the shared library."""
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    common = [nvcc, "-std=c++17", "-O3", "-lineinfo", "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"),
              "-I", CSRC, "-gencode", "arch=compute_100a,code=sm_100a"]
    if verbose:
        common += ["-Xptxas", "-v"]
    procs = []
    objs = []
    for src in SOURCES:
        obj = os.path.join(objdir, os.path.splitext(src)[0] + ".o")
        objs.append(obj)
        cmd = common + ["-x", "cu", "-c", os.path.join(CSRC, src), "-o", obj]
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = False
    for src, pr in procs:
        out, _ = pr.communicate()
        if pr.returncode != 0 or verbose:
            sys.stderr.write(f"--- {src}\n{out}\n")
        failed |= pr.returncode != 0
    if failed:
        raise RuntimeError("nvcc failed")
    link = [nvcc, "-shared", "-o", LIB] + objs + ["-gencode", "arch=compute_100a,code=sm_100a", "-lcudart"]
    subprocess.run(link, check=True)
    for source, module in (("native_module.c", NATIVE), ("paged_calls.c", PAGED)):
        subprocess.run([os.environ.get("CC", "gcc"), "-O2", "-Wall", "-shared", "-fPIC", "-I", sysconfig.get_paths()["include"],
                        "-I", os.path.join(ROOT, "include"), os.path.join(CSRC, source), "-o", module, "-L", HERE,
                        "-l:libheatkv.so", "-Wl,-rpath,$ORIGIN"], check=True)
    return LIB


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv))
