"""Build libkvec.so (HIP, gfx950) in-tree with hipcc, and the binding's marshalling module."""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(HERE, "libkvec.so")
BIND = os.path.join(HERE, "_kvec_bind.so")
BUILD_DIR = os.path.join(ROOT, "_build")

# (source, object name, extra flags): the step kernel is instantiated once per
# (dtype, head_dim) pair, in parallel translation units
SOURCES = [("kvec_api.hip", "kvec_api", []), ("kvec_pipeline.hip", "kvec_pipeline", []),
           ("kvec_decode.hip", "kvec_decode", []), ("kvec_serve_api.hip", "kvec_serve_api", []),
           ("kvec_prefill.hip", "kvec_prefill", []), ("kvec_append.hip", "kvec_append", []),
           ("kvec_paged_decode.hip", "kvec_paged_decode", []),
           ("kvec_paged_evict.hip", "kvec_paged_evict", [])] + [
    ("kvec_step_inst.hip", f"kvec_step_{tt.lower()}_d{d}{'_long' if long == 'true' else ''}",
     [f"-DKVEC_INST_TT={tt}", f"-DKVEC_INST_D={d}", f"-DKVEC_INST_LONG={long}"])
    for tt, long in (("BF16", "false"), ("F32", "false"), ("BF16", "true")) for d in (64, 128)]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # packed fp32 VALU ops stay disabled in all device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", INCLUDE, "-I", CSRC,
]


def _compile(item) -> str:
    src, name, extra = item
    obj = os.path.join(BUILD_DIR, name + ".o")
    cmd = [HIPCC, *FLAGS, *extra, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stdout}\n{r.stderr}")
    return obj


def build_binding() -> str:
    """The compiled marshalling module of the Python binding (host code, against torch's headers)."""
    import sysconfig

    import torch
    base = os.path.dirname(torch.__file__)
    tmp = BIND + ".tmp"
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", INCLUDE,
           "-isystem", os.path.join(base, "include"),
           "-isystem", os.path.join(base, "include", "torch", "csrc", "api", "include"),
           "-isystem", os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include"),
           "-isystem", sysconfig.get_paths()["include"],
           os.path.join(CSRC, "kvec_bind.cpp"), "-o", tmp,
           "-L", os.path.join(base, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{cmd[0]} failed for kvec_bind.cpp:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, BIND)
    return BIND


def build(verbose: bool = True) -> str:
    os.makedirs(BUILD_DIR, exist_ok=True)
    workers = max(1, min(len(SOURCES), int(os.environ.get("MAX_JOBS", os.cpu_count() or 1))))
    with cf.ThreadPoolExecutor(max_workers=workers) as ex:
        binding = ex.submit(build_binding)
        objs = list(ex.map(_compile, SOURCES))
        binding.result()
    tmp = LIB + ".tmp"
    r = subprocess.run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", tmp],
                       capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    if verbose:
        print(f"built {LIB}", file=sys.stderr)
    return LIB


if __name__ == "__main__":
    build()
