"""Build libbdcommit.so and libbdcache.so in-tree with nvcc for sm_103a.

libbdcommit.so holds the sources of csrc/, libbdcache.so those of csrc/cache/;
each exports the C ABI of its headers under include/ only.
Each translation unit (CUDA .cu, host-only C++ .cpp) is compiled in
parallel, then linked into its shared library (static CUDA runtime, no
link-time dependency on libcuda: the tensor-map encoder is fetched through the
runtime's driver entry point).
A stamp of the sources and flags skips the build when nothing changed.
"""

from __future__ import annotations

import hashlib
import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "libbdcommit.so")
LIB_CHECKS = os.path.join(PKG, "libbdcommit_checks.so")
CSRC_CACHE = os.path.join(CSRC, "cache")
LIB_CACHE = os.path.join(PKG, "libbdcache.so")

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ARCH + [
    "-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-Xcompiler", "-O3",
    "--expt-relaxed-constexpr", "-I" + INCLUDE, "-I" + CSRC,
]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libbdcommit")


def _sources(src_dir=CSRC):
    return sorted(os.path.join(src_dir, f) for f in os.listdir(src_dir) if f.endswith((".cu", ".cpp")))


def _stamp(nvcc: str, extra, src_dir=CSRC) -> str:
    h = hashlib.sha256()
    h.update(" ".join([nvcc] + NVCC_FLAGS + list(extra)).encode())
    files = _sources(src_dir) + sorted(
        os.path.join(d, f) for d in {CSRC, src_dir} for f in os.listdir(d) if f.endswith((".cuh", ".h"))
    ) + sorted(os.path.join(INCLUDE, f) for f in os.listdir(INCLUDE) if f.endswith(".h"))
    for f in files:
        h.update(f.encode())
        with open(f, "rb") as fh:
            h.update(fh.read())
    return h.hexdigest()


def build(verbose: bool = False, force: bool = False, extra_flags=(), checks: bool = False) -> str:
    """Compile every source and link libbdcommit.so and libbdcache.so; returns the path of libbdcommit.so.

    checks=True builds the bounds-checked variant instead (-DBD_CHECKS:
    device-side index checks that set a status bit rather than access out of
    range) as libbdcommit_checks.so, in its own build directory
    (libbdcache.so has no such variant: it checks the page numbers it is given in every build)."""
    extra_flags = list(extra_flags)
    if checks:
        return _build_one(CSRC, BUILD + "_checks", LIB_CHECKS, "bd_*", verbose, force, extra_flags + ["-DBD_CHECKS"])
    with ThreadPoolExecutor(max_workers=2) as ex:
        libs = [ex.submit(_build_one, CSRC, BUILD, LIB, "bd_*", verbose, force, extra_flags),
                ex.submit(_build_one, CSRC_CACHE, os.path.join(BUILD, "cache"), LIB_CACHE, "bdkv_*", verbose, force,
                          extra_flags)]
        return [f.result() for f in libs][0]


def _build_one(src_dir, build_dir, lib, symbols, verbose, force, extra_flags) -> str:
    nvcc = _nvcc()
    os.makedirs(build_dir, exist_ok=True)
    stamp_file = os.path.join(build_dir, "build.stamp")
    stamp = _stamp(nvcc, extra_flags, src_dir)
    if not force and os.path.exists(lib) and os.path.exists(stamp_file):
        with open(stamp_file) as f:
            if f.read().strip() == stamp:
                return lib

    def compile_one(src):
        obj = os.path.join(build_dir, os.path.splitext(os.path.basename(src))[0] + ".o")
        cmd = [nvcc] + NVCC_FLAGS + list(extra_flags) + ["-c", src, "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}:\n{r.stdout}\n{r.stderr}")
        if verbose and (r.stdout or r.stderr):
            sys.stderr.write(r.stdout + r.stderr)
        return obj

    srcs = _sources(src_dir)
    with ThreadPoolExecutor(max_workers=min(8, len(srcs))) as ex:
        objs = list(ex.map(compile_one, srcs))
    tmp = lib + ".tmp"
    exports = os.path.join(build_dir, "exports.map")
    with open(exports, "w") as f:
        f.write("{ global: %s; local: *; };\n" % symbols)  # only the C ABI is visible
    cmd = [nvcc] + ARCH + ["-shared", "-cudart", "static", "-Xlinker", "--version-script=" + exports,
                           "-o", tmp] + objs + ["-ldl"]  # libdl: the NVTX trace ranges load a tracer on demand
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, lib)
    with open(stamp_file, "w") as f:
        f.write(stamp)
    return lib


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv, force="-f" in sys.argv))
