"""Build ``libgoldy.so`` (the C-ABI library) in-tree for sm_103a.

Plain nvcc/g++ invocations, one object per translation unit, compiled in
parallel: ``planner.cpp`` (host C++), ``runtime.cu`` (launch manager),
``noalloc.cu`` (the entry point with a compiled-in scratch array),
``kernels.cu`` once per GO-Kernel kind (``-DGOLDY_KIND=k``), the layer
operators (``linear.cu``, ``repack.cu``, ``bias_grad.cu``, ``layernorm.cu``,
``router.cu``, ``route.cu``, ``residual_norm.cu``, ``keep8.cu``),
``residual_norm_kernels.cu`` once per direction, type and row layout, and
``linear_kernels.cu`` once per pass and activation.  Objects go to
``_build/`` next to this file and the library to
``paper_2409_02227_gb300/libgoldy.so``; both are git-ignored.  A rebuild is
skipped when the library is newer than every source and header.
"""
from __future__ import annotations

import concurrent.futures as cf
import glob
import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libgoldy.so")
NUM_KINDS = 11
# (pass, activation) of the linear-layer kernels; the weight gradient has none
LINEAR_KERNELS = [(k, a) for k in range(2) for a in range(5)] + [(2, 0)]

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def _nvcc() -> str:
    cand = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(cand):
        raise RuntimeError("nvcc not found")
    return cand


def _sources_mtime() -> float:
    files = glob.glob(os.path.join(CSRC, "*")) + glob.glob(os.path.join(INCLUDE, "*.h"))
    files.append(os.path.abspath(__file__))
    return max(os.path.getmtime(f) for f in files)


def _jobs(ptxas_verbose: bool):
    nvcc = _nvcc()
    common = ["-std=c++17", "-O3", "-Xcompiler", "-fPIC", "-I", CSRC, "-I", INCLUDE]
    cu = [nvcc] + common + ARCH + ["-lineinfo"]
    if ptxas_verbose:
        cu += ["-Xptxas", "-v"]
    jobs = []
    jobs.append(("planner", ["g++", "-std=c++17", "-O2", "-ffp-contract=off", "-fPIC", "-Wall", "-I", CSRC, "-I", INCLUDE,
                             "-c", os.path.join(CSRC, "planner.cpp")]))
    jobs.append(("runtime", cu + ["-c", os.path.join(CSRC, "runtime.cu")]))
    jobs.append(("noalloc", cu + ["-c", os.path.join(CSRC, "noalloc.cu")]))
    jobs.append(("ewise", cu + ["-c", os.path.join(CSRC, "ewise.cu")]))
    for name in ("linear", "repack", "bias_grad", "layernorm", "router", "route", "residual_norm", "keep8"):
        jobs.append((name, cu + ["-c", os.path.join(CSRC, name + ".cu")]))
    for direction in ("forward", "backward"):
        for kind in ("bf16", "f32"):
            for mode in range(3):
                name = f"residual_norm_{direction}_{kind}_{mode}"
                jobs.append((name, cu + [f"-DGOLDY_NORM_KERNEL={name}", f"-DGOLDY_NORM_F32={int(kind == 'f32')}",
                                         f"-DGOLDY_NORM_BACKWARD={int(direction == 'backward')}",
                                         f"-DGOLDY_NORM_MODE=RowMode({mode})", "-c",
                                         os.path.join(CSRC, "residual_norm_kernels.cu")]))
    for k, a in LINEAR_KERNELS:
        jobs.append((f"linear_kernels_p{k}_a{a}", cu + [f"-DGOLDY_LINEAR_PASS={k}", f"-DGOLDY_LINEAR_ACT={a}", "-c",
                                                        os.path.join(CSRC, "linear_kernels.cu")]))
    for k in range(NUM_KINDS):
        jobs.append((f"kernels_k{k}", cu + [f"-DGOLDY_KIND={k}", "-c", os.path.join(CSRC, "kernels.cu")]))
    return jobs


def build(force: bool = False, verbose: bool = False, ptxas_verbose: bool = False) -> str:
    """Compile and link; returns the library path."""
    if not force and os.path.exists(LIB) and os.path.getmtime(LIB) >= _sources_mtime():
        return LIB
    os.makedirs(BUILD, exist_ok=True)
    jobs = _jobs(ptxas_verbose)

    def run(job):
        name, cmd = job
        obj = os.path.join(BUILD, name + ".o")
        proc = subprocess.run(cmd + ["-o", obj], capture_output=True, text=True)
        return name, obj, proc

    workers = max(1, min(len(jobs), os.cpu_count() or 4))
    objs = []
    errors = []
    with cf.ThreadPoolExecutor(workers) as ex:
        for name, obj, proc in ex.map(run, jobs):
            if verbose or ptxas_verbose:
                sys.stderr.write(proc.stdout + proc.stderr)
            if proc.returncode != 0:
                errors.append(f"--- {name} ---\n{proc.stdout}{proc.stderr}")
            objs.append(obj)
    if errors:
        raise RuntimeError("build failed:\n" + "\n".join(errors))
    tmp = LIB + f".tmp{os.getpid()}"
    link = [_nvcc(), "-shared"] + ARCH + objs + ["-o", tmp]
    proc = subprocess.run(link, capture_output=True, text=True)
    if proc.returncode != 0:
        raise RuntimeError("link failed:\n" + proc.stdout + proc.stderr)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv,
                ptxas_verbose="--ptxas" in sys.argv))
