"""Builds libocs.so (hand-written HIP for gfx950) in-tree with hipcc, and the Python side of its most frequent calls with g++."""
import os
import subprocess
import sysconfig

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libocs.so")
CALLS = os.path.join(_HERE, "_rows_call.so")
SOURCES = ["ocs_api.hip", "reduce.hip", "select.hip", "quantize.hip", "qa_split.hip", "clip_search.hip", "qgemm.hip", "row_grids.hip",
           "qgemm_rows.hip", "token_logprobs.hip", "calib.hip"]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-ffp-contract=off",                      # no fused multiply-add: rounding as written
    "-fno-gpu-flush-denormals-to-zero",       # fp32 denormals behave as on the host
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def build_library(verbose=False):
    """Compile every HIP source into paper_1901_09504_amd/libocs.so.  Always recompiles."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    cmd = [hipcc, *HIPCC_FLAGS, *[os.path.join(CSRC, s) for s in SOURCES], "-o", LIB]
    if verbose:
        print(" ".join(cmd))
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in res.stdout.splitlines()
                    if "packed-fp32-ops' is not a recognized feature" not in l)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + out)
    if verbose and out.strip():
        print(out)
    build_calls(verbose)
    return LIB


def build_calls(verbose=False):
    """Compile paper_1901_09504_amd/_rows_call.so, which finds libocs.so beside itself."""
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-I" + sysconfig.get_paths()["include"],
           os.path.join(CSRC, "rows_call.cpp"), "-o", CALLS, "-L" + _HERE, "-l:libocs.so", "-Wl,-rpath,$ORIGIN"]
    if verbose:
        print(" ".join(cmd))
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if res.returncode != 0:
        raise RuntimeError("g++ failed:\n" + res.stdout)
    return CALLS


if __name__ == "__main__":
    print(build_library(verbose=True))
