"""Sizes at the limits of the 4-bit attention's plan: what is too large is refused without arithmetic
that overflows on the way (CPU, under UndefinedBehaviorSanitizer)."""
from test_host_sanitizers_rope_kv4 import _build, _run, pytestmark  # noqa: F401

SIZES = """
import sys
from paper_2609_36757_amd import fastvr
fastvr.LIB_PATH = sys.argv[1]
n = 1 << 24
refused = 0
#       B, H, Hkv, Nq, d, cache_len, chunk_len, window
for c in ((1 << 20, 65535, 65535, 1, 128, n, n, -1), (2147483647, 16, 16, 1, 128, n, n, -1), (2147483647, 32, 1, 1, 64, n, 1, 5),
          (1, 65535, 65535, 1 << 15, 128, n, 1, -1), (1, 65535, 1, 32768, 64, n, n - 1, 0), (1 << 15, 64, 1, 1 << 15, 128, n, n, -1),
          (1, 1, 1, 2147483647, 128, n, 1, n), (64, 1, 1, 1 << 30, 64, n, 1 << 62, 1 << 62), (1 << 23, 1, 1, 1, 64, n, n, -1),
          (1, 1, 1, 1, 128, n, 1 << 62, (1 << 63) - 1), (1 << 10, 64, 8, 1, 128, n, 1, n), (2147483647, 1, 1, 32, 128, 0, 1, -1)):
    try:
        assert 0 <= fastvr.kv4_attn_workspace(*c) <= 64 << 20, c
    except fastvr.FastVRError as e:
        assert e.status == fastvr.ERR_UNSUPPORTED, (c, e)
        refused += 1
assert refused >= 4
print("sizes done")
"""


def test_largest_sizes(tmp_path):
    lib = str(tmp_path / "libfastvr_hostcheck.so")
    _build(lib, ["host_stubs.cpp", "host_stubs_rope_kv4.cpp"])
    assert "sizes done" in _run([SIZES, lib])
