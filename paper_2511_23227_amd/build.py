"""Compile the HIP sources into paper_2511_23227_amd/libpcpp.so for gfx950 (hipcc cross-compiles without a GPU)."""
from __future__ import annotations

import contextlib
import fcntl
import os
import re
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libpcpp.so")
CALLS_DIR = HERE                                       # of the host code that checks tensors and makes outputs in the short calls
PROBE_LIB = os.path.join(HERE, "libpcpp_probe.so")     # the benchmark's peak-rate probe, outside the library's interface

# file -> extra flags.  The search kernels must not contract a*b+c into an FMA: the inclusion test
# is a fixed binary64 operation sequence shared with the CPU oracle by convention.
SOURCES = {
    "pcpp_api.hip": [],
    "scan.hip": [],
    "build_triplets.hip": ["-ffp-contract=off"],
    "spatial_order.hip": [],
    "mvmr_generic.hip": [],
    # MFMA results in ordinary vector registers: other instructions read them next
    "mvmr_weight.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
    "mvmr_rows_tile.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
    "mvmr_rows_pc.hip": [],
    "tune.hip": [],
    "act_pack.hip": [],
    "block_norm.hip": [],
    "log_probs.hip": [],
    "rows_api.hip": [],
    "dropout.hip": [],
    "group_norm.hip": [],
    "mx_pack.hip": [],
    "mx_product.hip": [],
    "pointwise_api.hip": [],
}

COMMON = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-Wall", "-Wno-unused-function",
          "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
          "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _compile(name: str, extra) -> str:
    src = os.path.join(CSRC, name)
    obj = os.path.join(OBJ, name + ".o")
    cmd = ["hipcc", "-c", src, "-o", obj] + COMMON + list(extra)
    r = subprocess.run(cmd, capture_output=True, text=True)
    noise = "packed-fp32-ops' is not a recognized feature"
    err = "\n".join(l for l in r.stderr.splitlines() if noise not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {name}:\n{err}")
    if err.strip():
        sys.stderr.write(err + "\n")
    return obj


def _calls_need() -> str | None:
    """What this machine lacks to compile the Python calls, or None.  The library itself needs none of it."""
    try:
        import torch
    except ImportError as e:
        return f"torch ({e})"
    if shutil.which("g++") is None:
        return "g++"
    headers = (os.path.join(sysconfig.get_paths()["include"], "Python.h"),
               os.path.join(os.path.dirname(os.path.abspath(torch.__file__)), "include", "torch", "csrc", "autograd", "python_variable.h"))
    return next((h for h in headers if not os.path.exists(h)), None)


def calls_lib() -> str:
    """The compiled side of the Python calls that fits this Python and this torch, whose binary interfaces it uses."""
    import torch
    return os.path.join(CALLS_DIR, re.sub(r"[^\w.-]", "_", f"_torch_calls.{sys.implementation.cache_tag}-torch{torch.__version__}") + ".so")


@contextlib.contextmanager
def _alone():
    """One build of this folder at a time, among processes and threads: they write the same intermediate files."""
    os.makedirs(OBJ, exist_ok=True)
    with open(os.path.join(OBJ, "lock"), "w") as lock:
        fcntl.flock(lock, fcntl.LOCK_EX)                # (given back when the file is closed)
        yield


def build_calls() -> str:
    """The compiled side of the Python calls (host code against this torch's and Python's headers)."""
    with _alone():
        return _build_calls()


def _build_calls() -> str:
    missing = _calls_need()
    if missing:
        raise RuntimeError(f"the compiled side of the Python calls cannot be built without {missing}")
    import torch
    root = os.path.dirname(os.path.abspath(torch.__file__))
    lib = calls_lib()
    tmp = lib + ".tmp"
    cmd = ["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden", "-Wall", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
           "-I", os.path.join(ROOT, "include"), "-isystem", os.path.join(root, "include"), "-isystem", os.path.join(root, "include", "torch", "csrc", "api", "include"),
           "-isystem", sysconfig.get_paths()["include"], os.path.join(CSRC, "torch_calls.cpp"), "-o", tmp,
           "-L", os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-ldl"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed for torch_calls.cpp:\n{r.stderr}")
    os.replace(tmp, lib)
    return lib


def build(verbose: bool = False) -> str:
    """The library, then the compiled side of the Python calls, which is left out, with a note, where torch, g++ or the headers are missing."""
    with _alone():
        return _build(verbose)


def _build(verbose: bool) -> str:
    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(lambda kv: _compile(*kv), SOURCES.items()))
    tmp = LIB + ".tmp"
    subprocess.run(["hipcc", "-shared", "-fPIC", "--offload-arch=gfx950", "-o", tmp] + objs, check=True)
    os.replace(tmp, LIB)
    probe = _compile("peak_probe.hip", [])
    tmp = PROBE_LIB + ".tmp"
    subprocess.run(["hipcc", "-shared", "-fPIC", "--offload-arch=gfx950", "-o", tmp, probe], check=True)
    os.replace(tmp, PROBE_LIB)
    missing = _calls_need()
    if missing:
        sys.stderr.write(f"the compiled side of the Python calls is not built: it needs {missing}\n")
    else:
        _build_calls()
    if verbose:
        print("built", LIB)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
