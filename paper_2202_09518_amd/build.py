"""Build libnmfmu.so (HIP, gfx950) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libnmfmu.so")
SOURCES = ["nmfmu_dense.hip", "nmfmu_pairs.hip", "nmfmu_csr.hip", "nmfmu_api.hip",
           "nmfmu_ragged_bf16.hip", "nmfmu_ragged_f16.hip", "nmfmu_ragged_f32.hip", "nmfmu_ragged_api.hip",
           "nmfmu_rows.hip", "nmfmu_route.hip", "nmfmu_product8.hip", "nmfmu_routed_api.hip"]
HEADERS = [os.path.join(CSRC, h) for h in ("nmfmu_internal.h", "nmfmu_device.h", "nmfmu_ragged_internal.h", "nmfmu_ragged_device.h",
                                           "nmfmu_ragged_kernels.h", "nmfmu_routed_internal.h", "nmfmu_routed_device.h")] + \
          [os.path.join(ROOT, "include", h) for h in ("nmfmu.h", "nmfmu_test.h", "nmfmu_ragged.h", "nmfmu_routed.h")]
HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-command-line-argument",
]


def sources():
    return [os.path.join(CSRC, s) for s in SOURCES]


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = sources() + HEADERS
    return any(os.path.getmtime(d) > t for d in deps)


def build(verbose: bool = False) -> str:
    """Compile every HIP source for gfx950 and link the shared library."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    objs = []
    procs = []
    for src in sources():
        obj = src[:-4] + ".o"
        cmd = [hipcc, *HIPCC_FLAGS, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", src, "-o", obj]
        if verbose:
            print(" ".join(cmd))
        procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    for cmd, p in procs:
        out, _ = p.communicate()
        out = "\n".join(l for l in out.splitlines() if "packed-fp32-ops" not in l)
        if p.returncode != 0:
            raise RuntimeError("hipcc failed: " + " ".join(cmd) + "\n" + out)
        if verbose and out.strip():
            print(out)
    cmd = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs]
    subprocess.check_call(cmd)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
