"""Compile the HIP libraries for gfx950 into paper_2602_08798_amd/: libcryptogen_hip.so, the evaluator, and
libcryptogen_requests.so, which calls it."""
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
SRC = os.path.join(HERE, "csrc", "cryptogen.hip")
LIB = os.path.join(HERE, "libcryptogen_hip.so")
DEPS = [SRC] + [os.path.join(HERE, "csrc", f) for f in ("kernels.hpp", "tables.hpp", "modarith.hpp")] + [
    os.path.join(os.path.dirname(HERE), "include", "cryptogen_bench.h"),
    os.path.join(os.path.dirname(HERE), "include", "cryptogen.h")]
REQ_SRC = os.path.join(HERE, "csrc", "requests.hip")
REQ_LIB = os.path.join(HERE, "libcryptogen_requests.so")
REQ_DEPS = [REQ_SRC, LIB] + [os.path.join(HERE, "csrc", f) for f in ("requests.hpp", "kernels.hpp", "tables.hpp", "modarith.hpp")] + [
    os.path.join(os.path.dirname(HERE), "include", f) for f in ("cryptogen_requests.h", "cryptogen.h")]

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-ffp-contract=off",                      # products and sums must round separately (explicit fma only)
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


# The second library finds the first beside it, or as already loaded under this name.  Its kernels are its own: hidden.
LINK = ["-Wl,-soname,libcryptogen_hip.so"]
REQ_LINK = ["-fvisibility=hidden", "-Wl,-soname,libcryptogen_requests.so", "-L" + HERE, "-lcryptogen_hip", "-Wl,-rpath,$ORIGIN"]


def _compile(src, lib, deps, force, extra):
    if force or not os.path.exists(lib) or any(os.path.getmtime(lib) < os.path.getmtime(d) for d in deps):
        subprocess.run(["hipcc"] + FLAGS + ["-o", lib, src] + extra, check=True)


def build(force: bool = True, extra=()) -> str:
    _compile(SRC, LIB, DEPS, force, LINK + list(extra))
    _compile(REQ_SRC, REQ_LIB, REQ_DEPS, force, REQ_LINK + list(extra))
    return LIB


if __name__ == "__main__":
    print(build(force=True, extra=sys.argv[1:]))
