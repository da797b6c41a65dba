"""Build libfastvr.so in-tree with hipcc for gfx950.

    python -m paper_2609_36757_amd.build

Every HIP source is compiled with packed-FP32 instruction selection disabled
(``-target-feature -packed-fp32-ops``).  A build with a kernel that spills vector registers or
uses scratch memory is refused: an attention kernel that spilled accumulators gave wrong sums in
some lanes (a reload under a partial execution mask), besides being slow."""
from __future__ import annotations

import os
import re
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB_NAME = "libfastvr.so"
LIB_PATH = os.path.join(PKG, LIB_NAME)
SOURCES = ["chunk_attn_fwd.hip", "chunk_attn_bwd.hip", "kv_append.hip", "one_step.hip", "tiles.hip",
           "rope.hip", "kv4_cache.hip", "kv4_attn.hip", "fastvr_api.cpp", "geometry.cpp"]
ARCH = "gfx950"


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found (ROCm is required to build libfastvr.so)")


def compile_cmd(out: str) -> list[str]:
    return [hipcc(), f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-shared",
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            "-Wall", "-Wno-unused-function",
            "-I", INCLUDE, "-I", CSRC,
            *[os.path.join(CSRC, s) for s in SOURCES], "-o", out]


RESOURCES = "-Rpass-analysis=kernel-resource-usage"  # what each kernel takes, as remarks


def spilling(remarks: str) -> list[str]:
    """The kernels that spill vector registers or use scratch memory, from the compiler's remarks."""
    bad = []
    for kernel in remarks.split("remark: Function Name: ")[1:]:
        used = re.findall(r"(?: VGPRs Spill|ScratchSize \[bytes/lane\]): (\d+)", kernel)
        if any(int(n) for n in used):
            bad.append(kernel.split()[0])
    return bad


def build(verbose: bool = False) -> str:
    tmp = LIB_PATH + f".tmp{os.getpid()}"
    cmd = compile_cmd(tmp) + [RESOURCES]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    spills = spilling(res.stderr)
    if res.returncode != 0 or spills:
        if os.path.exists(tmp):
            os.unlink(tmp)
        if res.returncode != 0:
            raise RuntimeError(f"hipcc failed ({res.returncode}):\n{res.stdout}\n{res.stderr}")
        raise RuntimeError(f"kernels that spill vector registers or use scratch memory: {', '.join(spills)}")
    os.replace(tmp, LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
