"""Builds in-tree: libemaslice.so with nvcc for sm_100a (cross-compiles without a GPU), and the extension module that fills in
the device-driven calls' arguments from torch tensors, with the host compiler. The library needs neither torch nor the extension."""
from __future__ import annotations

import importlib.util
import os
import re
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libemaslice.so")
SOURCES = ["slice.cpp", "copy_kernels.cu", "layer_kernel.cu", "noalloc.cu", "paged_api.cpp", "paged_tables.cu", "paged_decode.cu", "paged_tree.cu", "paged_pages.cu"]
HEADERS = ["kernels.h", "ptx.cuh", "tcgen05.cuh", "attention_tiles.cuh", os.path.join("..", "..", "include", "emaslice.h")]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    return "nvcc"


TORCH_CALLS = os.path.join(HERE, "_torch_calls.so")
TORCH_CALLS_FOR = os.path.join(HERE, "_torch_calls.for.txt")   # the Python and the torch it was built for (git-ignored)
TORCH_SOURCES = ["torch_calls.cpp"]


def _older(product: str, sources) -> bool:
    if not os.path.exists(product):
        return True
    t = os.path.getmtime(product)
    return any(os.path.getmtime(d) > t for d in [os.path.join(CSRC, f) for f in sources] + [os.path.abspath(__file__)])


def needs_build() -> bool:
    return _older(LIB, SOURCES + HEADERS)


def _torch_dir():
    """Where torch is installed (it is not imported), or None."""
    spec = importlib.util.find_spec("torch")
    return spec.submodule_search_locations[0] if spec and spec.submodule_search_locations else None


def torch_calls_wanted() -> str:
    """The Python and the torch that the extension has to be built for here."""
    with open(os.path.join(_torch_dir(), "version.py")) as f:
        version = re.search(r"__version__ = '([^']+)'", f.read())
    return f"{sysconfig.get_config_var('SOABI')} torch {version.group(1) if version else 'unknown'}"


def torch_calls_built_for() -> str:
    """And those that it was built for; empty if that is not known."""
    if not os.path.exists(TORCH_CALLS_FOR):
        return ""
    with open(TORCH_CALLS_FOR) as f:
        return f.read().strip()


def build_torch_calls(force: bool = False, verbose: bool = False) -> str:
    torch = _torch_dir()
    if torch is None:
        raise RuntimeError("torch is not installed: the device-driven calls on tensors need it (the library itself does not)")
    wanted = torch_calls_wanted()
    if not force and not _older(TORCH_CALLS, TORCH_SOURCES + HEADERS[-1:]) and torch_calls_built_for() == wanted:
        return TORCH_CALLS
    # nvcc's host compiler, with the C++ runtime that torch's libraries use (a compiler set to link its own in does not do).
    cmd = ["g++", "-std=c++17", "-O2", "-fPIC", "-shared", "-Wall", "-I" + sysconfig.get_paths()["include"],
           "-isystem", os.path.join(torch, "include"), "-isystem", os.path.join(torch, "include", "torch", "csrc", "api", "include")]
    cmd += [os.path.join(CSRC, f) for f in TORCH_SOURCES]
    cmd += ["-o", TORCH_CALLS, "-L" + os.path.join(torch, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"]
    if os.path.exists(TORCH_CALLS_FOR):
        os.remove(TORCH_CALLS_FOR)
    try:
        res = subprocess.run(cmd, capture_output=True, text=True)
    except OSError as e:
        raise RuntimeError(f"the host compiler cannot be run for _torch_calls.so: {e}") from e
    if verbose or res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
    if res.returncode != 0:
        raise RuntimeError("the host compiler failed building _torch_calls.so")
    with open(TORCH_CALLS_FOR, "w") as f:
        f.write(wanted + "\n")
    return TORCH_CALLS


RESOURCES = os.path.join(HERE, "libemaslice.resources.txt")   # ptxas' report of the last build (git-ignored)


def build_library(force: bool = False, verbose: bool = False) -> str:
    if not force and not needs_build() and os.path.exists(RESOURCES):
        return LIB
    cmd = [_nvcc(), "-std=c++17", "-O3", "-lineinfo", "-gencode", "arch=compute_100a,code=sm_100a",
           "-Xcompiler", "-fPIC,-Wall,-Wno-unused-function", "-Xptxas", "-v", "-shared", "-o", LIB]
    cmd += [os.path.join(CSRC, f) for f in SOURCES]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed building libemaslice.so")
    with open(RESOURCES, "w") as f:
        f.write(res.stdout + res.stderr)
    return LIB


def build(force: bool = False, verbose: bool = False) -> str:
    """Both. Without the extension the library is of use all the same, so that what keeps that one from being built is told, and
    raised by the first call that needs it (or by build_torch_calls)."""
    build_library(force, verbose)
    try:
        build_torch_calls(force, verbose)
    except RuntimeError as e:
        sys.stderr.write(f"the device-driven calls on tensors are not available: {e}\n")
    return LIB


def kernel_resources() -> dict:
    """What ptxas reported for every kernel of the last build: registers per thread, bytes of stack
    frame, bytes of spill stores and loads, keyed by the kernel's (mangled) name. The layer kernel runs
    352 threads per CTA at the register limit of one CTA per SM; a change that makes it spill, or
    that makes the compiler keep a copy of its 1 KB parameter block on every thread's stack, costs
    several per cent of its bandwidth, and this report is where that shows without a GPU."""
    build_library()
    out, name = {}, None
    with open(RESOURCES) as f:
        for line in f:
            m = re.search(r"Compiling entry function '([^']+)'", line)
            if m:
                name = m.group(1)
                out[name] = {}
                continue
            if name is None:
                continue
            m = re.search(r"(\d+) bytes stack frame, (\d+) bytes spill stores, (\d+) bytes spill loads", line)
            if m and "stack" not in out[name]:
                out[name].update(stack=int(m.group(1)), spill_stores=int(m.group(2)), spill_loads=int(m.group(3)))
            m = re.search(r"Used (\d+) registers", line)
            if m:
                out[name]["registers"] = int(m.group(1))
                name = None
    return out


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
