"""Compile the HIP sources for gfx950 into paper_2503_00245_amd/libmoe_mi355x.so.

hipcc cross-compiles without a GPU.  Each .hip file becomes an object (compiled in
parallel), then one shared library exporting the C ABI of include/moe.h.
"""
import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libmoe_mi355x.so")
SOURCES = ["api.hip", "route.hip", "permute.hip", "combine.hip", "expert_gemv.hip", "expert_gemv_one.hip", "expert_gemm.hip", "expert_gemm_f32.hip",
           "expert_gemm_pp.hip", "expert_gemm_few.hip",
           "metrics.hip", "route_scored.hip", "mxfp4_rows.hip", "mxfp4_experts.hip", "mxfp4_few.hip", "mxfp4_gemm.hip", "mxfp4_stream.hip"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fvisibility=hidden",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         # scalar arguments at the head of a kernel's list arrive in registers instead of by a load: 0.2-0.5 us a launch
         "-mllvm", "-amdgpu-kernarg-preload-count=16",
         "-Wall", "-Wno-unused-command-line-argument",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _hipcc():
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if c and (os.path.isabs(c) and os.path.exists(c) or not os.path.isabs(c)):
            return c
    return "hipcc"


def _compile(src):
    obj = os.path.join(OBJ, src.replace(".hip", ".o"))
    cmd = [_hipcc(), *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{err}")
    return obj, err


def build(verbose: bool = False) -> str:
    os.makedirs(OBJ, exist_ok=True)
    with ThreadPoolExecutor(max_workers=7) as ex:
        results = list(ex.map(_compile, SOURCES))
    if verbose:
        for _, err in results:
            if err.strip():
                print(err)
    objs = [o for o, _ in results]
    cmd = [_hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", LIB]
    subprocess.run(cmd, check=True)
    return LIB


def ensure_built() -> str:
    """Build only when no library is there (tests, the smoke run and the benchmark call this;
    the binding itself never builds: a missing library is an error there)."""
    return LIB if os.path.exists(LIB) else build()


if __name__ == "__main__":
    print(build(verbose=True))
