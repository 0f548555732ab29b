"""Builds libcombo_b200.so (sm_100a) in-tree with nvcc."""
from __future__ import annotations

import os
import shutil
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "libcombo_b200.so")
OBJ = os.path.join(HERE, "build")
# sources, one object file each, and the headers they include beside the public one
HEADERS = {
    "combo_b200.cu": ("segment_aggregate.cuh", "select_peers.cuh", "divergence.cuh", "pull_aggregate.cuh", "host_common.h"),
    "group_norm.cu": ("host_common.h", "step_common.cuh"),
    "grouped_linear.cu": ("host_common.h", "step_common.cuh", "tensor_core.cuh"),
    "grad_clip.cu": ("host_common.h", "step_common.cuh"),
}
SOURCES = [os.path.join(CSRC, f) for f in HEADERS]
PUBLIC = os.path.join(INCLUDE, "combo_b200.h")


def nvcc_path() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def _depends(src: str) -> list[str]:
    return [src, PUBLIC] + [os.path.join(CSRC, h) for h in HEADERS[os.path.basename(src)]]


def _newer(target: str, files) -> bool:
    """Whether `target` is missing or older than one of `files`."""
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(f) > t for f in files)


def is_stale() -> bool:
    return any(_newer(LIB, _depends(src)) for src in SOURCES)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not is_stale():
        return LIB
    tmp = LIB + ".%d.tmp" % os.getpid()
    os.makedirs(OBJ, exist_ok=True)
    arch = ["-gencode", "arch=compute_100a,code=sm_100a"]
    running, objects, spare = [], [], []
    for src in SOURCES:
        obj = os.path.join(OBJ, os.path.basename(src) + ".o")
        objects.append(obj)
        if force or _newer(obj, _depends(src)):
            part = obj + ".%d.tmp.o" % os.getpid()
            spare.append((part, obj))
            running.append(subprocess.Popen(
                [nvcc_path()] + arch + ["-lineinfo", "-O3", "-std=c++17", "-Xptxas", "-v" if verbose else "-warn-spills",
                                        "-Xcompiler", "-fPIC", "-c", "-o", part, src]))
    if any([p.wait() for p in running]):
        for part, _ in spare:
            if os.path.exists(part):
                os.remove(part)
        raise RuntimeError("nvcc failed")
    for part, obj in spare:
        os.replace(part, obj)
    subprocess.check_call([nvcc_path()] + arch + ["-shared", "-Xcompiler", "-fPIC", "-o", tmp] + objects)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
