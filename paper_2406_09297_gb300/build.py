"""Builds libmlkv.so in place (nvcc, sm_103a only).

Translation units compile in parallel; the ptxas report (registers, spills, shared memory) of
each kernel is kept in _build/ptxas.log.
"""
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libmlkv.so")
INCLUDE = os.path.join(ROOT, "include")

NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc" if os.path.exists(
    "/usr/local/cuda/bin/nvcc") else "nvcc")
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
COMMON = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-I", INCLUDE, "-I", CSRC]
SOURCES = ["mlkv_kernels.cu", "mlkv_decode_tc.cu", "mlkv_prefill.cu", "mlkv_merge.cu",
           "mlkv_stage.cu", "mlkv_host.cpp", "mlkv_noalloc.cu", "mlkv_measure.cu", "mlkv_norm_rope.cu",
           "mlkv_q4.cu", "mlkv_q4_decode.cu", "mlkv_q4_host.cpp", "mlkv_pieces.cu", "mlkv_blocks.cu",
           "mlkv_evict.cu", "mlkv_long_host.cpp"]


def _sources():
    return [os.path.join(CSRC, s) for s in SOURCES]


def _deps():
    deps = _sources() + [os.path.join(CSRC, "mlkv_internal.h"), os.path.join(CSRC, "mlkv_device.cuh"),
                         os.path.join(CSRC, "mlkv_tcgen05.cuh"), os.path.join(CSRC, "mlkv_host.h"),
                         os.path.join(CSRC, "mlkv_q4.h"), os.path.join(CSRC, "mlkv_cache.h"),
                         os.path.join(CSRC, "mlkv_long.h"), os.path.join(CSRC, "mlkv_topk.cuh"),
                         os.path.join(CSRC, "mlkv_plan.h"),
                         os.path.join(INCLUDE, "mlkv.h"),
                         os.path.abspath(__file__)]
    return deps


def needs_build():
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(p) > t for p in _deps())


def _compile(src):
    obj = os.path.join(BUILD, os.path.basename(src) + ".o")
    cmd = [NVCC, *ARCH, *COMMON, "-c", src, "-o", obj]
    if src.endswith(".cu"):
        cmd += ["-Xptxas", "-v"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"nvcc failed for {src}:\n{r.stdout}\n{r.stderr}")
    return obj, r.stderr


def build(force=False, verbose=False):
    if not force and not needs_build():
        return LIB
    os.makedirs(BUILD, exist_ok=True)
    with ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        results = list(ex.map(_compile, _sources()))
    with open(os.path.join(BUILD, "ptxas.log"), "w") as f:
        for _, log in results:
            f.write(log)
    tmp = LIB + ".tmp"
    cmd = [NVCC, *ARCH, "-shared", "-o", tmp, *[o for o, _ in results], "-cudart", "static"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    if verbose:
        for _, log in results:
            sys.stderr.write(log)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
