"""Builds ``librdfft.so`` (the HIP kernels and the C ABI) in-tree for gfx950, and ``_binding.so``, the Python module
that hands torch tensors to it.

Run ``python -m paper_2511_01385_amd.build`` or call :func:`build`.  Objects go to
``paper_2511_01385_amd/_build/``; the shared library lands next to this file.
"""

from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "librdfft.so")

SOURCES = ["bca_block_bf16.hip", "bca_block_f16.hip", "bca_block_f32.hip", "bca_store_bf16.hip", "bca_store_f16.hip", "bca_store_f32.hip", "rdfft_kernels.hip", "rdfft_hc_kernels.hip", "bca_kernels.hip", "bca_multipass.hip", "layout_kernels.hip", "mixed_kernels.hip", "act8_kernels.hip", "norm_kernels.hip", "linear_bf16.hip", "linear_f16.hip", "linear_f32.hip", "linear.hip", "capi.cpp", "capi_dense.cpp", "twiddles.cpp"]

BINDING = os.path.join(PKG, "_binding.so")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"

# Packed FP32 instructions (v_pk_*_f32) are disabled for every HIP object: the compiler
# would otherwise form them from float2 arithmetic, and the kernels are written for the
# scalar FP32 forms.
COMMON = [
    "-O3",
    "-std=c++17",
    "-fPIC",
    "-fvisibility=hidden",
    f"--offload-arch={ARCH}",
    "-Xclang",
    "-target-feature",
    "-Xclang",
    "-packed-fp32-ops",
    "-munsafe-fp-atomics",
    f"-I{INCLUDE}",
    f"-I{CSRC}",
    "-Wno-unused-command-line-argument",
]


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    # capi.cpp and capi_dense.cpp call the HIP runtime, so they are compiled as HIP; twiddles.cpp is plain C++
    lang = ["-x", "c++"] if src == "twiddles.cpp" else ["-x", "hip"]
    cmd = [HIPCC, *COMMON, *lang, "-c", os.path.join(CSRC, src), "-o", obj]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{res.stderr}")
    return obj


def _build_binding() -> bool:
    """Compiles csrc/binding.cpp (plain C++) against torch's headers and the built library, which it finds next to itself.

    By hipcc too: no other compiler is needed.  Without torch there is nothing to bind (False): C callers have their library.
    """
    try:
        import torch
    except ImportError:
        return False
    root = os.path.dirname(torch.__file__)
    cmd = [
        HIPCC, "-x", "c++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
        f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
        f"-I{INCLUDE}", f"-I{root}/include", f"-I{root}/include/torch/csrc/api/include",
        f"-I{sysconfig.get_paths()['include']}", os.path.join(CSRC, "binding.cpp"), "-o", BINDING + ".tmp",
        "-x", "none", LIB, f"-L{root}/lib", "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-Wl,-rpath,$ORIGIN",
    ]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed on binding.cpp:\n{res.stderr}")
    shutil.move(BINDING + ".tmp", BINDING)
    return True


def build(verbose: bool = True) -> str:
    """Compile every source and link ``librdfft.so``; returns the library path."""
    if not os.path.exists(HIPCC):
        raise RuntimeError(f"hipcc not found at {HIPCC}")
    os.makedirs(BUILD, exist_ok=True)
    jobs = min(len(SOURCES), max(1, min(16, os.cpu_count() or 1)))
    with ThreadPoolExecutor(max_workers=jobs) as ex:
        objs = list(ex.map(_compile, SOURCES))
    tmp = LIB + ".tmp"
    cmd = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-Wl,-soname,librdfft.so", "-o", tmp, *objs]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"link failed:\n{res.stderr}")
    shutil.move(tmp, LIB)
    bound = _build_binding()
    if verbose:
        print(f"built {LIB}" + ("" if bound else " (without its Python module: there is no torch)"), file=sys.stderr)
    return LIB


if __name__ == "__main__":
    build()
