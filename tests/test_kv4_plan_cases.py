"""The kernels that the calls of tests/kv4_plan_cases.py reach (CPU)."""
import os
import shutil
import subprocess

import pytest

from kv4_plan_cases import PARITY, VISIBILITY

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_36757_amd", "csrc")


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_calls_reach_the_kernels_they_are_for(tmp_path):
    exe = str(tmp_path / "kv4_plan_print")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, os.path.join(ROOT, "tests", "kv4_plan_print.cpp"),
                    "-o", exe], check=True, timeout=300)
    calls = PARITY + VISIBILITY
    lines = "".join(f"{c.B} {c.H} {c.Hkv} {c.Nq} {c.d} {c.n} {c.L} {c.W}\n" for c in calls)
    out = subprocess.run([exe], input=lines, capture_output=True, text=True, timeout=60, check=True).stdout.splitlines()
    assert out == [f"{c.tiles} {c.split} {c.join}" for c in calls]


def test_every_pair_of_kernels_has_a_call():
    for d in (64, 128):
        for tiles in (1, 2, 4):
            for split, join in (("none", None), ("split", "group"), ("split", "wave")):
                assert any((c.tiles, c.split, c.join, c.d) == (tiles, split, join, d) for c in PARITY), (tiles, split, join, d)
        for tiles in (2, 4):
            assert any((c.tiles, c.split, c.join, c.d) == (tiles, "tail", "wave", d) for c in PARITY)
    # a last row tile that is not full, in split tiles of every height
    for tiles in (1, 2, 4):
        assert any(c.tiles == tiles and c.split != "none" and c.Nq * c.H // c.Hkv % (16 * tiles) for c in PARITY)
