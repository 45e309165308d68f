"""Builds the C-ABI library ``libciar.so`` in-tree with hipcc for gfx950, and the native Python module ``_step.so`` on it."""
from __future__ import annotations

import os
import subprocess
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libciar.so")
STEP = os.path.join(HERE, "_step.so")
STEP_SOURCE = "ciar_torch.cpp"
SOURCES = ["ciar_stream.hip", "ciar_rows.hip", "ciar_short.hip", "ciar_radius.hip", "ciar_finish.hip", "ciar_heads.hip", "ciar_loss.hip", "ciar_aux.hip", "ciar_interhead.hip", "ciar_plan.hip", "ciar_rotary.hip", "ciar_attention.hip", "ciar_logits.hip", "ciar_api.cpp", "ciar_step.cpp"]
HEADERS = ["ciar_internal.h", "ciar_host.h", "ciar_step.h", "ciar_device.h", "ciar_stream.h", os.path.join("..", "..", "include", "ciar.h")]

# Packed-FP32 instructions are switched off for every device compile of this library.
HIPCC_FLAGS = ["-O3", "-std=c++17", "-fPIC", "--offload-arch=gfx950",
               "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
               "-Wall", "-Wno-unused-function"]


def stale() -> bool:
    if not os.path.exists(LIB) or not os.path.exists(STEP):
        return True
    t = min(os.path.getmtime(LIB), os.path.getmtime(STEP))
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS + [STEP_SOURCE]] + [os.path.abspath(__file__)]
    return any(os.path.getmtime(d) > t for d in deps)


def torch_dir() -> str:
    import torch
    return os.path.dirname(torch.__file__)


def compile_step(verbose: bool = False) -> str:
    """The native module's object: host code only, against torch's headers."""
    obj, torch_include = os.path.join(CSRC, os.path.splitext(STEP_SOURCE)[0] + ".o"), os.path.join(torch_dir(), "include")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-w", "-D__HIP_PLATFORM_AMD__", "-DUSE_ROCM",
           "-I" + torch_include, "-I" + os.path.join(torch_include, "torch", "csrc", "api", "include"), "-I/opt/rocm/include",
           "-I" + sysconfig.get_paths()["include"], "-c", os.path.join(CSRC, STEP_SOURCE), "-o", obj]
    if verbose:
        print(" ".join(cmd))
    subprocess.run(cmd, check=True, stdout=subprocess.DEVNULL if not verbose else None,
                   stderr=subprocess.PIPE if not verbose else None)
    return obj


def build(force: bool = True, verbose: bool = False) -> str:
    """Compile and link.  ``force=False`` skips the work when the library is newer than its sources."""
    if not force and not stale():
        return LIB
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    def compile_one(src: str) -> str:
        obj = os.path.join(CSRC, os.path.splitext(src)[0] + ".o")
        cmd = [hipcc, *HIPCC_FLAGS, "-x", "hip", "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd))
        subprocess.run(cmd, check=True, stdout=subprocess.DEVNULL if not verbose else None,
                       stderr=subprocess.PIPE if not verbose else None)
        return obj

    with ThreadPoolExecutor(max_workers=min(len(SOURCES) + 1, os.cpu_count() or 1, 8)) as pool:
        step = pool.submit(compile_step, verbose)
        objs = list(pool.map(compile_one, SOURCES))
        step_obj = step.result()
    cmd = [hipcc, "-shared", "-fPIC", "--offload-arch=gfx950", "-o", LIB, *objs]
    if verbose:
        print(" ".join(cmd))
    subprocess.run(cmd, check=True)
    lib_dir = os.path.join(torch_dir(), "lib")
    cmd = ["g++", "-shared", "-o", STEP, step_obj, "-L" + HERE, "-l:libciar.so", "-L" + lib_dir, "-ltorch_python", "-ltorch",
           "-ltorch_cpu", "-lc10", "-lc10_hip", "-Wl,-rpath,$ORIGIN"]
    if verbose:
        print(" ".join(cmd))
    subprocess.run(cmd, check=True)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
