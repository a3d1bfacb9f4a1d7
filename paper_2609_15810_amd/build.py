"""Build the HIP library libvcattn.so for gfx950 (hipcc), in-tree next to this file, and the
standalone matrix-core probe mfma_probe (the measured ceilings bench.py reports beside the roofline)."""
from __future__ import annotations

import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(ROOT, "_build")
LIB = os.path.join(HERE, "libvcattn.so")
SOURCES = ["api.hip", "prep.hip", "forward.hip", "group.hip", "block_api.hip", "norm_rope.hip", "cross_fwd.hip",
           "cross_bwd.hip"]
HEADERS = ["vc_common.hpp", "vc_internal.hpp", "cross_common.hpp", "lanes.hpp"]
PROBE = os.path.join(HERE, "mfma_probe")

# -ffp-contract=off: every fp32 operation that decides a stored code is a single IEEE operation,
# fused multiply-adds are written explicitly. Packed fp32 instructions are disabled.
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _compile(src: str) -> str:
    obj = os.path.join(OBJ, src.replace(".hip", ".o"))
    cmd = ["hipcc", *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stderr}")
    return obj


def _probe() -> str:
    tmp = PROBE + ".tmp%d" % os.getpid()
    cmd = ["hipcc", "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang",
           "-packed-fp32-ops", os.path.join(CSRC, "mfma_probe.hip"), "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for mfma_probe.hip:\n{r.stderr}")
    os.replace(tmp, PROBE)
    return PROBE


def build() -> str:
    """Compile every source and link the shared library, and build the probe (always rebuilds)."""
    os.makedirs(OBJ, exist_ok=True)
    with ThreadPoolExecutor(len(SOURCES) + 1) as ex:
        probe = ex.submit(_probe)
        objs = list(ex.map(_compile, SOURCES))
        probe.result()
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = ["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build())
