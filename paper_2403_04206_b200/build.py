"""In-tree build of libgrawa.so (nvcc, sm_100a only)."""
from __future__ import annotations

import os
import shutil
import subprocess

_HERE = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_HERE)
CSRC = os.path.join(_HERE, "csrc")
LIB_PATH = os.path.join(_HERE, "libgrawa.so")
DEBUG_LIB_PATH = os.path.join(_HERE, "libgrawa_debug_bounds.so")
TRACE_LIB_PATH = os.path.join(_HERE, "libgrawa_trace.so")
SOURCES = [os.path.join(CSRC, "grawa.cu")]
HEADERS = [os.path.join(CSRC, "kernels.cuh"), os.path.join(CSRC, "center_pull_bulk.cuh"), os.path.join(CSRC, "kernels_16bit.cuh"), os.path.join(CSRC, "center_pull_staged_any.cuh"),
           os.path.join(CSRC, "host_common.h"), os.path.join(_ROOT, "include", "grawa.h")]
# The replica operators have no debug or trace code of their own: one object, linked into every variant.
OPS_OBJECT = os.path.join(_HERE, "_build", "replica_ops.o")
OPS_SOURCE = os.path.join(CSRC, "replica_ops.cu")
OPS_HEADERS = [os.path.join(CSRC, h) for h in ("replica_common.cuh", "replica_host.h", "dropout.cuh", "layernorm.cuh", "gated_ffn.cuh", "host_common.h")] + [
    os.path.join(_ROOT, "include", "grawa.h")]

# The binding's marshaller of pointer tables (a CPython module that reads torch tensors).
MARSHAL_PATH = os.path.join(_HERE, "_marshal.so")
MARSHAL_SOURCE = os.path.join(CSRC, "marshal.cpp")

# No fast-math: arithmetic is IEEE but for the approximate functions that the sources call by name (the activations of the gated
# feed-forward product, the reciprocal root of layer norm).
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-shared", "-Xcompiler", "-fPIC"]


def _nvcc() -> str:
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found: libgrawa.so cannot be built and there is no fallback path")
    return exe


def is_stale(path: str = LIB_PATH) -> bool:
    if not os.path.exists(path):
        return True
    t = os.path.getmtime(path)
    return any(os.path.getmtime(p) > t for p in SOURCES + HEADERS + [OPS_SOURCE] + OPS_HEADERS)


def _run(cmd) -> str:
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("compilation failed:\n" + " ".join(cmd) + "\n" + res.stdout + res.stderr)
    return res.stderr


def _build_ops(force: bool, verbose: bool = False) -> str:
    """The object of the replica operators, compiled when missing or older than its sources."""
    if force or not os.path.exists(OPS_OBJECT) or any(os.path.getmtime(p) > os.path.getmtime(OPS_OBJECT) for p in [OPS_SOURCE] + OPS_HEADERS):
        os.makedirs(os.path.dirname(OPS_OBJECT), exist_ok=True)
        tmp = OPS_OBJECT + f".tmp{os.getpid()}.o"
        flags = [f for f in NVCC_FLAGS if f != "-shared"] + (["-Xptxas", "-v"] if verbose else [])
        log = _run([_nvcc()] + flags + ["-c", "-o", tmp, OPS_SOURCE])
        if verbose:
            print(log)
        os.replace(tmp, OPS_OBJECT)
    return OPS_OBJECT


def build_marshal(force: bool = False) -> str:
    """Compiles the marshaller when missing or older than its source; returns its path."""
    if force or not os.path.exists(MARSHAL_PATH) or os.path.getmtime(MARSHAL_SOURCE) > os.path.getmtime(MARSHAL_PATH):
        import sysconfig
        import torch
        base = os.path.dirname(torch.__file__)
        tmp = MARSHAL_PATH + f".tmp{os.getpid()}"
        _run([shutil.which("g++") or "g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I" + os.path.join(base, "include"),
              "-I" + os.path.join(base, "include", "torch", "csrc", "api", "include"), "-I" + sysconfig.get_paths()["include"],
              MARSHAL_SOURCE, "-o", tmp, "-L" + os.path.join(base, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"])
        os.replace(tmp, MARSHAL_PATH)
    return MARSHAL_PATH


def _build_variant(path: str, define: str, force: bool) -> str:
    if force or is_stale(path):
        tmp = path + f".tmp{os.getpid()}"
        _run([_nvcc()] + NVCC_FLAGS + [define, "-o", tmp] + SOURCES + [_build_ops(False)])
        os.replace(tmp, path)
    return path


def build(force: bool = False, verbose: bool = False, debug_bounds: bool = False, trace: bool = False) -> str:
    """Compile the CUDA library when missing or older than its sources; returns its path.
    debug_bounds: the variant whose kernels check their global accesses against the plan;
    trace: the variant whose kernels stamp the device timer (see grawa_trace_read)."""
    if debug_bounds:
        return _build_variant(DEBUG_LIB_PATH, "-DGRAWA_DEBUG_BOUNDS", force)
    if trace:
        return _build_variant(TRACE_LIB_PATH, "-DGRAWA_TRACE", force)
    if force or is_stale():
        tmp = LIB_PATH + f".tmp{os.getpid()}"
        ops = _build_ops(force, verbose)
        log = _run([_nvcc()] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-o", tmp] + SOURCES + [ops])
        if verbose:
            print(log)
        os.replace(tmp, LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    print(build(force=True, verbose=True))
