"""Builds libfcsim.so (CUDA kernels + C ABI) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libfcsim.so")
HOST_SOURCE = os.path.join(CSRC, "fcsim.cu")
KERNEL_SOURCE = os.path.join(CSRC, "fcsim_step_kernels.cu")   # compiled once per policy
N_KERNEL_POLICIES = 7
KV_SOURCE = os.path.join(CSRC, "fcsim_kv.cu")                  # the paged key-value cache
KV_ATTEND_SOURCE = os.path.join(CSRC, "fcsim_kv_attend.cu")    # its attention, compiled once per pair of types
KV_PREFILL_SOURCE = os.path.join(CSRC, "fcsim_kv_prefill.cu")  # and of several tokens, the same
N_KV_TYPES = 2 * 4                                             # objects of the two
SOURCES = [HOST_SOURCE, KERNEL_SOURCE, KV_SOURCE, KV_ATTEND_SOURCE, KV_PREFILL_SOURCE]
HEADERS = [os.path.join(CSRC, "fcsim_device.cuh"), os.path.join(ROOT, "include", "fcsim.h"),
           os.path.join(CSRC, "fcsim_kv_device.cuh"), os.path.join(CSRC, "fcsim_kv_attend.cuh"),
           os.path.join(CSRC, "fcsim_kv_prefill.cuh"),
           os.path.join(ROOT, "include", "fcsim_kv.h")]
OBJ_DIR = os.path.join(HERE, "_build")


def _stale(lib: str = LIB) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    return any(os.path.getmtime(f) > t for f in SOURCES + HEADERS)


LIB_CHECKED = os.path.join(HERE, "libfcsim_checked.so")


def build(force: bool = False, verbose: bool = False, checked: bool = False) -> str:
    """Compile if the sources are newer than the library; returns the library path.
    ``checked`` builds the index-checked diagnostic variant (libfcsim_checked.so)."""
    if checked:
        if not force and not _stale(LIB_CHECKED):
            return LIB_CHECKED
        return _compile(LIB_CHECKED, verbose, ["-DFCSIM_CHECKED"])
    if not force and not _stale():
        return LIB
    return _compile(LIB, verbose, [])


def _compile(lib: str, verbose: bool, extra) -> str:
    """One object per policy's step kernels plus the host file, compiled side by side, then linked.  Every object
    is a module of its own to the compiler, so the result does not depend on how many cores built it."""
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tag = os.path.splitext(os.path.basename(lib))[0]
    os.makedirs(OBJ_DIR, exist_ok=True)
    common = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC,-Wall", "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    if verbose:
        common += ["-Xptxas", "-v"]
    extra = list(extra)
    jobs = [(HOST_SOURCE, extra, os.path.join(OBJ_DIR, f"{tag}_host.o"))]
    for pol in range(N_KERNEL_POLICIES):
        jobs.append((KERNEL_SOURCE, extra + [f"-DFCSIM_KERNEL_POLICY={pol}"], os.path.join(OBJ_DIR, f"{tag}_policy{pol}.o")))
    # the cache's objects are the same in both builds: the checked one takes those that are there
    kv = [(KV_SOURCE, [], os.path.join(OBJ_DIR, "kv.o"))]
    for source, name in ((KV_ATTEND_SOURCE, "kv_attend"), (KV_PREFILL_SOURCE, "kv_prefill")):
        for types in range(N_KV_TYPES // 2):
            kv.append((source, [f"-DFCSIM_KV_TYPES={types}"], os.path.join(OBJ_DIR, f"{name}{types}.o")))
    jobs += kv
    there = {obj for _, _, obj in kv if extra and not _stale(obj)}

    def one(job):
        src, defs, obj = job
        if obj in there:
            return subprocess.CompletedProcess([], 0, "", "")
        return subprocess.run(common + defs + ["-c", src, "-o", obj], capture_output=True, text=True)

    with ThreadPoolExecutor(max_workers=min(len(jobs), os.cpu_count() or 1)) as pool:
        results = list(pool.map(one, jobs))
    for (src, defs, obj), r in zip(jobs, results):
        if r.stdout or r.stderr:
            sys.stderr.write(f"[{os.path.basename(obj)}]\n{r.stdout}{r.stderr}")
        if r.returncode != 0:
            raise subprocess.CalledProcessError(r.returncode, r.args)
    subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-o", lib + ".tmp"]
                   + [obj for _, _, obj in jobs], check=True)
    os.replace(lib + ".tmp", lib)
    return lib


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, checked="--checked" in sys.argv))
