"""Builds libgva.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import hashlib
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libgva.so")
PROBE_LIB = os.path.join(HERE, "libgva_probe.so")      # the benchmark's read-only streaming probe (not part of the C ABI)
_SHARED = ["gva_common.cuh", "gva_rope.cuh", "gva_decode_mma.cuh", "gva_handle.cuh", os.path.join("..", "..", "include", "gva.h")]
SOURCES = {   # source -> the headers it is compiled from
    "gva_api.cu": _SHARED + ["gva_small_kernels.cuh", "gva_decode_fma.cuh", "gva_decode_fp8.cuh", "gva_prefill.cuh", "gva_project.cuh"],
    "gva_compact.cu": _SHARED + ["gva_q4.cuh", "gva_q4_decode.cuh", "gva_weights.cuh", "gva_evict.cuh"],
}


def _newer(target: str, files) -> bool:
    """Whether target is there and no file is newer than it."""
    return os.path.exists(target) and all(os.path.getmtime(target) >= os.path.getmtime(f) for f in files if os.path.exists(f))


def _files(source: str):
    return [os.path.join(CSRC, f) for f in [source] + SOURCES[source]]


def _object(source: str, command) -> str:
    """The object of a source, named after the command that makes it, so that other flags never find it."""
    return os.path.join(CSRC, f"{source[:-3]}.{hashlib.sha256(' '.join(command).encode()).hexdigest()[:12]}.o")


def build(force: bool = False, verbose: bool = False) -> str:
    if os.environ.get("GVA_LIBRARY"):      # a prebuilt library was named explicitly: nothing to do
        return os.environ["GVA_LIBRARY"]
    if not force and all(_newer(LIB, _files(f)) for f in SOURCES):
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    arch = ["-gencode", "arch=compute_100a,code=sm_100a"]
    flags = arch + ["-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC"]
    if os.path.exists(os.path.join(CSRC, "gva_decode_mma.cuh")):
        flags.append("-DGVA_WITH_MMA")
    extra = os.environ.get("GVA_EXTRA_NVCC_FLAGS", "").split()   # e.g. tuning macros such as -DGVA_MMA_WPG64=1
    compile_ = [nvcc, "-c"] + flags + extra
    objects = {f: _object(f, compile_) for f in SOURCES}
    jobs = []                                                     # the sources are compiled side by side
    for f, obj in objects.items():
        if force or verbose or not _newer(obj, _files(f)):
            part = f"{obj[:-2]}.{os.getpid()}.o"                  # takes its name once it is whole
            cmd = compile_ + (["-Xptxas", "-v"] if verbose else []) + [os.path.join(CSRC, f), "-o", part]
            jobs.append((subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True), part, obj))
    failed = False
    for job, part, obj in jobs:
        said = job.communicate()[0]
        if verbose or job.returncode != 0:
            sys.stderr.write(said)
        if job.returncode == 0:
            os.replace(part, obj)
        else:
            failed = True
            if os.path.exists(part):
                os.unlink(part)
    if failed:
        raise RuntimeError("nvcc failed building libgva.so")
    link = subprocess.run([nvcc] + arch + extra + ["-shared"] + list(objects.values()) + ["-o", LIB], capture_output=True, text=True)
    if link.returncode != 0:
        sys.stderr.write(link.stdout + link.stderr)
        raise RuntimeError("nvcc failed linking libgva.so")
    return LIB


def build_probe(force: bool = False) -> str:
    """Builds the benchmark's read-only streaming probe (csrc/stream_probe.cu) into its own shared object."""
    src = os.path.join(CSRC, "stream_probe.cu")
    if not force and os.path.exists(PROBE_LIB) and os.path.getmtime(PROBE_LIB) >= os.path.getmtime(src):
        return PROBE_LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-shared", "-Xcompiler", "-fPIC",
           src, "-o", PROBE_LIB]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("nvcc failed building libgva_probe.so")
    return PROBE_LIB


if __name__ == "__main__":
    build_probe(force=True)
    print(build(force=True, verbose="-v" in sys.argv))
