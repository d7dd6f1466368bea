"""Builds ``libpwlq.so`` (the C-ABI CUDA library) in-tree with nvcc for sm_100a, and the PyTorch module of
the training calls with the host compiler."""
from __future__ import annotations

import os
import subprocess
import sys
import warnings

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libpwlq.so")
PEAK_LIB = os.path.join(HERE, "libpwlq_peak.so")     # FP32 micro-benchmark, loaded by bench.py only
PEAK_SOURCES = ["fp32_peak.cu"]
CALLS_LIB = os.path.join(HERE, "_pwlq_calls.so")     # imported as a Python module
CALLS_SOURCE = "pwlq_calls.cpp"
SOURCES = ["pwlq_api.cu", "pwlq_absmax.cu", "pwlq_search.cu", "pwlq_quantize.cu",
           "pwlq_noalloc.cu", "pwlq_select.cu", "pwlq_search2.cu", "pwlq_bias.cu", "pwlq_rowmap.cu",
           "pwlq_act8.cu", "pwlq_block_norm.cu", "pwlq_weight_grad.cu", "pwlq_train_api.cu",
           "pwlq_w4.cu", "pwlq_w4_linear_f32.cu", "pwlq_w4_linear_bf16.cu", "pwlq_w4_linear_f16.cu",
           "pwlq_w4_moe.cu", "pwlq_w4_moe_route.cu", "pwlq_w4_moe_f32.cu", "pwlq_w4_moe_bf16.cu",
           "pwlq_w4_moe_f16.cu", "pwlq_w4_api.cu"]
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo",
    "-fmad=false",            # no implicit FMA contraction: every fused op is an explicit fmaf
    "--shared", "-Xcompiler", "-fPIC", "-cudart", "static",
    "--threads", "0",         # the source files are compiled side by side
]


def _stale(lib: str) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    deps += [os.path.join(HERE, "..", "include", "pwlq.h"), os.path.abspath(__file__)]
    return any(os.path.getmtime(d) > t for d in deps)


def _nvcc(sources, lib: str, verbose: bool) -> None:
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + \
          [os.path.join(CSRC, s) for s in sources] + ["-o", lib]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    if verbose:
        print(res.stderr)


def _calls(verbose: bool) -> None:
    import sysconfig

    import torch
    root = os.path.dirname(torch.__file__)
    cuda = os.path.join(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")), "..")
    include = [os.path.join(root, "include"), os.path.join(root, "include/torch/csrc/api/include"),
               sysconfig.get_paths()["include"], os.path.join(cuda, "include")]
    # the system compiler: the module has to share one libstdc++ with PyTorch
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared",
           "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI)]
    cmd += [a for i in include for a in ("-isystem", i)]
    cmd += [os.path.join(CSRC, CALLS_SOURCE), "-o", CALLS_LIB, "-L" + os.path.join(root, "lib"),
            "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("g++ failed:\n" + res.stdout + res.stderr)
    if verbose:
        print(res.stderr)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compiles the library (and the benchmark's FP32 micro-benchmark) if a source is newer, and the module of
    the training calls.  That one alone needs PyTorch's and Python's headers: where it cannot be built, the
    library is complete all the same, a warning says why, and the training calls of the package raise."""
    if force or _stale(LIB):
        _nvcc(SOURCES, LIB, verbose)
    if force or _stale(PEAK_LIB):
        _nvcc(PEAK_SOURCES, PEAK_LIB, verbose)
    if force or _stale(CALLS_LIB):
        try:
            _calls(verbose)
        except (ImportError, OSError, RuntimeError) as e:
            if os.path.exists(CALLS_LIB):        # of other sources: it must not be loaded
                os.remove(CALLS_LIB)
            warnings.warn(f"the module of the training calls was not built: {e}")
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
