"""Build libgmc.so in-tree with nvcc for sm_103a (GB300).

    python -m paper_1905_12948_gb300.build [--force] [--verbose]

Each CUDA translation unit is compiled in parallel into ``_build/`` and linked
into ``paper_1905_12948_gb300/libgmc.so`` (static CUDA runtime); beside it
``_tokens.so``, the Python module of the operators on torch tensors, is compiled
against the torch that is installed (where there is none, or one without CUDA, the
library alone is built). Floating-point
flags keep one IEEE rounding per operation: no FMA contraction (-fmad=false on
the device, -ffp-contract=off on the host), no flush-to-zero, IEEE division.
"""
from __future__ import annotations

import argparse
import concurrent.futures
import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libgmc.so")
TOKENS = os.path.join(PKG, "_tokens.so")

SOURCES = ["gmc_api.cu", "gmc_topk.cu", "gmc_small.cu", "gmc_rbgs.cu", "gmc_noalloc.cu",
           "gmc_loss.cu", "gmc_policy.cu", "gmc_dropout.cu", "gmc_scores.cu", "gmc_ortho.cu"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-std=c++17", "-lineinfo", *ARCH,
         "-fmad=false", "-ftz=false", "-prec-div=true", "-prec-sqrt=true",
         "-Xcompiler", "-fPIC", "-Xcompiler", "-ffp-contract=off",
         "-I", INCLUDE, "-I", CSRC]


def nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def _headers():
    hs = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))]
    return hs + [os.path.join(INCLUDE, "gmc.h")]


def _stale(target, deps):
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def _tokens_command(cc: str, out: str):
    """The compiler's command for the Python module, and a line that tells what it was built for;
    None without a torch to build against."""
    import sysconfig

    try:
        import torch
    except ImportError:
        return None
    if torch.version.cuda is None:
        return None
    home = os.path.dirname(torch.__file__)
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(cc))), "include")
    abi = int(torch._C._GLIBCXX_USE_CXX11_ABI)
    lib = os.path.join(home, "lib")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={abi}",
           "-I", INCLUDE, "-I", os.path.join(home, "include"),
           "-I", os.path.join(home, "include", "torch", "csrc", "api", "include"),
           "-I", sysconfig.get_path("include"), "-I", cuda, os.path.join(CSRC, "binding.cpp"), "-o", out,
           "-L", lib, "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda", f"-Wl,-rpath,{lib}"]
    return cmd, f"{torch.__version__} {sys.version_info[:2]} {home}"


def build(force: bool = False, verbose: bool = False, extra_flags=()) -> str:
    os.makedirs(BUILD, exist_ok=True)
    cc = nvcc()
    headers = _headers()
    objs, jobs = [], []
    for src in SOURCES:
        s = os.path.join(CSRC, src)
        o = os.path.join(BUILD, src.replace(".cu", ".o"))
        objs.append(o)
        if force or _stale(o, [s, *headers, __file__]):
            jobs.append([cc, *FLAGS, *extra_flags, "-c", s, "-o", o])

    tokens, made_for = _tokens_command(cc, TOKENS + f".{os.getpid()}.tmp") or (None, "")
    stamp = os.path.join(BUILD, "tokens.txt")
    known = open(stamp).read() if os.path.exists(stamp) else ""
    if tokens and (force or known != made_for or _stale(TOKENS, [os.path.join(CSRC, "binding.cpp"), *headers, __file__])):
        jobs.append(tokens)

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        p = subprocess.run(cmd, capture_output=True, text=True)
        if p.returncode != 0:
            raise RuntimeError(f"{os.path.basename(cmd[0])} failed:\n{' '.join(cmd)}\n{p.stdout}\n{p.stderr}")
        if verbose and (p.stdout or p.stderr):
            print(p.stdout + p.stderr, flush=True)

    with concurrent.futures.ThreadPoolExecutor(max_workers=len(jobs) or 1) as ex:
        list(ex.map(run, jobs))
    if tokens in jobs:
        os.replace(tokens[tokens.index("-o") + 1], TOKENS)
        with open(stamp, "w") as f:
            f.write(made_for)
    if force or jobs or _stale(LIB, objs):
        run([cc, "-shared", *ARCH, "-o", LIB, *objs, "-cudart", "static"])
    return LIB


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__)
    ap.add_argument("--force", action="store_true")
    ap.add_argument("--verbose", action="store_true")
    ap.add_argument("--ptxas-info", action="store_true", help="print register / smem usage")
    a = ap.parse_args(argv)
    extra = ["-Xptxas", "-v"] if a.ptxas_info else []
    print(build(force=a.force or a.ptxas_info, verbose=a.verbose or a.ptxas_info, extra_flags=extra))


if __name__ == "__main__":
    sys.exit(main())
