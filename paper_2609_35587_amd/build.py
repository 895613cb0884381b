"""Build libhwsel.so (the HIP kernels and the C ABI) for gfx950 and _binding.so
(Python calls of it, host code against torch), in-tree.

Every translation unit is compiled with hipcc for gfx950 only; packed-fp32
instructions are disabled; the feature, evaluation and sampling units are also
compiled without multiply-add contraction, as is dropout's (their rounding steps
are part of their contract).
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libhwsel.so")
# measured ceilings for the benchmark's rooflines: a library of its own
CEIL_SRC, CEIL_LIB = "ceilings.hip", os.path.join(HERE, "libhwsel_ceilings.so")
BINDING_SRC, BINDING = "binding.cpp", os.path.join(HERE, "_binding.so")
ARCH = "gfx950"
SOURCES = ["api.hip", "catalogue.hip", "dropout.hip", "evaluate.hip", "features.hip", "forest.hip", "fp8.hip",
           "fp8_matmul.hip", "join.hip", "logprob.hip", "mlp.hip", "sample.hip", "scorers.hip", "select.hip"]
COMMON = ["-O3", "-std=c++20", "-fPIC", f"--offload-arch={ARCH}", "-fno-fast-math",
          "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
          "-Wall", "-Wno-unused-function", "-Wno-unknown-pragmas"]
PER_FILE = {"dropout.hip": ["-ffp-contract=off"], "features.hip": ["-ffp-contract=off"], "evaluate.hip": ["-ffp-contract=off"],
            "sample.hip": ["-ffp-contract=off"]}


def hipcc() -> str:
    return os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "bin", "hipcc")


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, src.replace(".hip", ".o"))
    cmd = [hipcc(), *COMMON, *PER_FILE.get(src, []), "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stderr}")
    if r.stderr.strip():
        sys.stderr.write(r.stderr)
    return obj


def _binding() -> None:
    import sysconfig

    import torch
    t = os.path.dirname(torch.__file__)
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    include = [os.path.join(t, "include"), os.path.join(t, "include", "torch", "csrc", "api", "include"),
               os.path.join(rocm, "include"), sysconfig.get_paths()["include"], os.path.join(os.path.dirname(HERE), "include")]
    tmp = BINDING + f".tmp{os.getpid()}"
    # (the defines that the runtime's and torch's own headers ask of a host compiler)
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-D__HIP_PLATFORM_AMD__", "-DUSE_ROCM",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", *[a for i in include for a in ("-isystem", i)],
           os.path.join(CSRC, BINDING_SRC), "-L" + os.path.join(t, "lib"), "-ltorch_python", "-ltorch_cpu", "-ltorch_hip", "-lc10_hip", "-lc10",
           "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode:
        raise RuntimeError(f"g++ failed for {BINDING_SRC}:\n{r.stderr}")
    if r.stderr.strip():
        sys.stderr.write(r.stderr)
    os.replace(tmp, BINDING)


def build(jobs: int = 8) -> str:
    os.makedirs(BUILD, exist_ok=True)
    with ThreadPoolExecutor(jobs) as ex:
        binding = ex.submit(_binding)
        objs = list(ex.map(_compile, SOURCES + [CEIL_SRC]))
        binding.result()
    ceil_obj = objs.pop()
    for out, parts in ((LIB, objs), (CEIL_LIB, [ceil_obj])):
        tmp = out + f".tmp{os.getpid()}"
        subprocess.run([hipcc(), "-shared", "-fPIC", f"--offload-arch={ARCH}", *parts, "-o", tmp], check=True)
        os.replace(tmp, out)
    return LIB


if __name__ == "__main__":
    print(build())
