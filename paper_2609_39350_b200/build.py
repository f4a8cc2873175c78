"""Builds libhap.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import subprocess

_DIR = os.path.dirname(os.path.abspath(__file__))
LIB = os.path.join(_DIR, "libhap.so")
LIB_CHECKED = os.path.join(_DIR, "libhap_checked.so")      # the same sources with -DHAP_CHECKED (self-checking kernels)
SOURCES = [os.path.join(_DIR, "csrc", "hap_api.cu"), os.path.join(_DIR, "csrc", "hap_operators.cu"),
           os.path.join(_DIR, "csrc", "hap_measure.cu"), os.path.join(_DIR, "csrc", "hap_tokens.cu")]
HEADERS = [os.path.join(_DIR, "csrc", "hap_device.cuh"), os.path.join(_DIR, "csrc", "hap_tree.cuh"),
           os.path.join(_DIR, "csrc", "hap_tree_host.h"), os.path.join(_DIR, "csrc", "hap_joint.cuh"),
           os.path.join(os.path.dirname(_DIR), "include", "hap.h")]
OPERATOR_HEADERS = [os.path.join(_DIR, "csrc", "hap_values.cuh"), os.path.join(_DIR, "csrc", "hap_launch.h"), os.path.join(_DIR, "csrc", "hap_products.cuh"), os.path.join(_DIR, "csrc", "hap_products_tc.cuh"),
                    os.path.join(_DIR, "csrc", "hap_products_experts.cuh"), os.path.join(_DIR, "csrc", "hap_products_few.cuh"), os.path.join(_DIR, "csrc", "hap_adamw.cuh"),
                    os.path.join(os.path.dirname(_DIR), "include", "hap.h")]

TOKEN_HEADERS = [os.path.join(_DIR, "csrc", "hap_values.cuh"), os.path.join(_DIR, "csrc", "hap_launch.h"), os.path.join(_DIR, "csrc", "hap_route.cuh"),
                 os.path.join(_DIR, "csrc", "hap_rows.cuh"), os.path.join(_DIR, "csrc", "hap_norm.cuh"), os.path.join(os.path.dirname(_DIR), "include", "hap.h")]

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "--fmad=false", "-std=c++17",
              "-shared", "-Xcompiler", "-fPIC"]


def is_stale(lib: str = LIB) -> bool:
    return _older(lib, SOURCES + HEADERS + OPERATOR_HEADERS + TOKEN_HEADERS)


def _older(target: str, inputs) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(f) > t for f in inputs)


def build_library(force: bool = False, verbose: bool = False, checked: bool = False) -> str:
    """Compile the library (or its self-checking variant) if it is missing or older than its sources; returns its path.
    Sources are compiled side by side, each into an object beside the library, and those that did not change are kept."""
    lib = LIB_CHECKED if checked else LIB
    if force or is_stale(lib):
        nvcc = os.environ.get("NVCC", "nvcc")
        more = [*(["-DHAP_CHECKED"] if checked else []), *(["-Xptxas", "-v"] if verbose else [])]
        objects, running = [], []
        for src, headers in zip(SOURCES, (HEADERS, OPERATOR_HEADERS, OPERATOR_HEADERS[-1:], TOKEN_HEADERS)):
            obj = lib[:-len(".so")] + "_" + os.path.basename(src)[:-len(".cu")] + ".o"
            objects.append(obj)
            if force or _older(obj, [src, *headers]):
                flags = [f for f in NVCC_FLAGS if f != "-shared"]
                running.append(subprocess.Popen([nvcc, *flags, *more, "-c", "-o", obj, src]))
        failed = [p.args for p in running if p.wait() != 0]
        if failed:
            raise subprocess.CalledProcessError(1, failed[0])
        subprocess.run([nvcc, *NVCC_FLAGS, "-o", lib, *objects], check=True)
    return lib
