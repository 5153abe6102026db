"""Compile the CUDA library in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

_PKG = os.path.dirname(os.path.abspath(__file__))
_CSRC = os.path.join(_PKG, "csrc")
_INCLUDE = os.path.join(os.path.dirname(_PKG), "include")
LIB_PATH = os.path.join(_PKG, "liblinfusion_attn.so")
# each source and the headers it includes
_SOURCES = {
    "linfusion_attn.cu": ["common.cuh", "split_kernels.cuh", "stream_kernels.cuh", "fused_kernels.cuh", "producer_kernels.cuh",
                          "padded_kernels.cuh", "linfusion_attn.h"],
    "attn_backward.cu": ["common.cuh", "backward_kernels.cuh", "backward_tc_kernels.cuh",
                         "backward_tc_wide_kernels.cuh", "packed_math.cuh", "host_util.h",
                         "linfusion_attn.h"],
    "block_ops.cu": ["common.cuh", "block_kernels.cuh", "packed_math.cuh", "host_checks.h", "host_util.h", "linfusion_attn.h",
                     "linfusion_block.h"],
    "pack8.cu": ["common.cuh", "pack8.cuh", "block_kernels.cuh", "packed_math.cuh", "host_checks.h", "host_util.h", "linfusion_attn.h",
                 "linfusion_block.h", "linfusion_layers.h"],
    "recurrence.cu": ["common.cuh", "recurrence_kernels.cuh", "column_sums.cuh", "pack8.cuh", "packed_math.cuh", "sigmoid.cuh", "host_checks.h", "host_util.h",
                      "linfusion_attn.h", "linfusion_block.h", "linfusion_layers.h"],
    "linear.cu": ["common.cuh", "linear_kernels.cuh", "column_sums.cuh", "handover.h", "pack8.cuh", "block_kernels.cuh", "packed_math.cuh", "sigmoid.cuh",
                  "host_checks.h", "host_util.h", "linfusion_attn.h", "linfusion_block.h", "linfusion_layers.h"],
}
CHECKED_LIB_PATH = os.path.join(_PKG, "liblinfusion_attn_checked.so")


def _mtime(name: str) -> float:
    return os.path.getmtime(os.path.join(_INCLUDE if name.startswith("linfusion_") and name.endswith(".h") else _CSRC, name))


def _newest_source_mtime() -> float:
    return max(_mtime(n) for source, headers in _SOURCES.items() for n in [source] + headers)


def build_library(force: bool = False, verbose: bool = False, checked: bool = False) -> str:
    """Build ``liblinfusion_attn.so`` next to this file if it is missing or stale; only the objects whose
    sources changed are compiled again.  ``checked=True`` builds ``liblinfusion_attn_checked.so`` instead:
    the same sources with -DLF_CHECKED, in which every global-memory address the split / cluster kernels
    compute is compared with the buffers of the call and an access outside them is counted and skipped
    (a debugging build, slower)."""
    out = CHECKED_LIB_PATH if checked else LIB_PATH
    if not force and os.path.exists(out) and os.path.getmtime(out) >= _newest_source_mtime():
        return out
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    flags = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-Xcompiler", "-fPIC"]
    if checked:
        flags += ["-DLF_CHECKED"]
    if verbose:
        flags += ["-Xptxas", "-v"]
    obj_dir = os.path.join(_PKG, "_build", "checked" if checked else "release")
    os.makedirs(obj_dir, exist_ok=True)

    def compile_one(source: str) -> str:
        obj = os.path.join(obj_dir, source[:-3] + ".o")
        newest = max(_mtime(n) for n in [source] + _SOURCES[source])
        if force or not os.path.exists(obj) or os.path.getmtime(obj) < newest:
            subprocess.run([nvcc, *flags, "-c", "-o", obj, os.path.join(_CSRC, source)], check=True)
        return obj

    with ThreadPoolExecutor(len(_SOURCES)) as pool:
        objects = list(pool.map(compile_one, _SOURCES))
    subprocess.run([nvcc, *flags, "-shared", "-o", out, *objects], check=True)
    return out


if __name__ == "__main__":
    print(build_library(force=True, verbose=True))
