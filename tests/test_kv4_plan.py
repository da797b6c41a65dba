"""The 4-bit attention's work plan (csrc/kv4_plan.h) on the CPU, and what its kernels compile to."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2609_36757_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_36757_amd", "csrc")


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_kv4_plan(tmp_path):
    exe = str(tmp_path / "kv4_plan_check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-Wall", "-Werror", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=all", "-I", CSRC, os.path.join(ROOT, "tests", "kv4_plan_check.cpp"), "-o", exe],
                   check=True, timeout=300)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]
    assert "cases ok" in r.stdout


@pytest.mark.parametrize("source,kernels", [("kv4_attn.hip", 10), ("kv4_cache.hip", 4), ("rope.hip", 48)])
def test_no_register_spills(tmp_path, source, kernels):
    """Every kernel keeps its vector registers: an attention kernel that spilled accumulators gave
    wrong values for some lanes, besides being slow."""
    cmd = build.compile_cmd(str(tmp_path / "x.o"))
    cmd = [a for a in cmd if not a.endswith((".hip", ".cpp")) and a != "-shared"]
    cmd[1:1] = ["-c", os.path.join(CSRC, source), "--offload-device-only", "-Rpass-analysis=kernel-resource-usage"]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    spills = [int(x) for x in re.findall(r" VGPRs Spill: (\d+)", r.stderr)]
    scratch = [int(x) for x in re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", r.stderr)]
    assert len(spills) == len(scratch) == kernels, (len(spills), len(scratch))
    assert not any(spills) and not any(scratch), (spills, scratch)
