"""Builds the CUDA library in-tree: paper_2601_21198_b200/libzipmoe.so (sm_100a only)."""
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libzipmoe.so")
SOURCES = ["zipmoe_host.cpp", "planner.cpp", "scheduler.cpp", "decode_kernel.cu", "ffn_kernels.cu", "recover_kernel.cu",
           "norm_kernel.cu", "router_kernel.cu", "resident_ffn_kernel.cu", "resident_few_kernel.cu", "group_kernel.cu",
           "quantize_kernel.cu", "grouped_matmul.cu", "grouped_few_kernel.cu",
           "grouped_wide_kernel.cu"]
HEADERS = ["zipmoe_format.h", "decode_device.cuh", "tile_geometry.h", "tensor_core.cuh", "resident.cuh", "resident_choice.h",
           "grouped.cuh", "grouped_launch.h", "grouped_choice.h", os.path.join(ROOT, "include", "zipmoe.h")]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "--use_fast_math",
              "-Xcompiler", "-fPIC,-O3,-Wall", "-shared", "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _nvcc():
    for c in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if c and (os.path.isabs(c) and os.path.exists(c) or not os.path.isabs(c)):
            return c
    return "nvcc"


def needs_build():
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, s) for s in SOURCES] + [h if os.path.isabs(h) else os.path.join(CSRC, h) for h in HEADERS]
    deps.append(os.path.abspath(__file__))
    return any(os.path.getmtime(d) > t for d in deps)


def build(force=False, verbose=False):
    """Compile every CUDA source for sm_100a into one shared library."""
    if not force and not needs_build():
        return LIB
    tmp = LIB + ".tmp%d" % os.getpid()
    extra = os.environ.get("ZIPMOE_NVCC_EXTRA", "").split()   # e.g. -DZIPMOE_WARPS=20 when tuning
    cmd = [_nvcc()] + NVCC_FLAGS + extra + (["-Xptxas", "-v"] if verbose else []) + \
          [os.path.join(CSRC, s) for s in SOURCES] + ["-o", tmp, "-lcudart", "-ldl"]
    subprocess.check_call(cmd)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
