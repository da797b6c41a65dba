"""The host layer of the rotary and 4-bit cache entry points under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU): every refusal of tests/test_abi_rope_kv4.py, and calls that pass all
checks and reach stand-in launchers.  A build of the layer without those launchers refuses the calls."""
import os
import subprocess
import sys

from test_host_sanitizers import CSRC, ENV_SAN, ROOT, SAN, _asan_runtime, pytestmark  # noqa: F401

VALID = """
import sys
from paper_2609_36757_amd import fastvr
fastvr.LIB_PATH = sys.argv[1]
want = int(sys.argv[2])
import test_abi_rope_kv4 as t
for raw, good, more in ((fastvr.rope_raw, t.ROPE, [dict(y=t.X), dict(x_fp32=1, y_fp32=1), dict(n_pairs=0, split1=0, split2=0, inv_freq=None),
                                                   dict(n_axes=3, split1=12, split2=22, pos_sb=48), dict(B=1, x_sb=0, y_sb=0)]),
                        (fastvr.kv4_append_raw, t.COPY, [dict(starts=t.ST, first=-5), dict(first=61), dict(v=t.KN)]),
                        (fastvr.kv4_read_raw, t.COPY, [dict(starts=t.ST), dict(k_st=512, k_sb=1536, v_st=512, v_sb=1536, v=t.KN + 512)]),
                        (fastvr.kv4_attn_raw, t.ATTN, [dict(lens=t.LENS, o_bf16=1, lse=None), dict(cache_len=0, workspace=None),
                                                       dict(chunk_len=1, window_chunks=7), dict(Nq=5000, q_sb=5000 * 512, o_sb=5000 * 512)])):
    for kw in [{}] + more:
        status = raw(*dict(good, **kw).values(), None)
        assert status == want, (raw.__name__, kw, status, fastvr.last_error())
        assert want == 0 or "no kernels" in fastvr.last_error()
print("valid calls done")
"""


def _build(lib, stubs):
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", *SAN, "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I",
                    os.path.join(ROOT, "include"), "-I", CSRC, os.path.join(CSRC, "fastvr_api.cpp"), os.path.join(CSRC, "geometry.cpp"),
                    *[os.path.join(ROOT, "tests", s) for s in stubs], "-o", lib], check=True, timeout=300)


def _run(args):
    env = dict(os.environ, LD_PRELOAD=_asan_runtime(), PYTHONPATH=os.pathsep.join((ROOT, os.path.join(ROOT, "tests"))), **ENV_SAN)
    r = subprocess.run([sys.executable, "-c", *args], cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    out = r.stdout[-3000:] + r.stderr[-3000:]
    assert r.returncode == 0 and "ERROR: AddressSanitizer" not in out and "runtime error" not in out, out
    return r.stdout


def test_layer_under_sanitizers(tmp_path):
    lib = str(tmp_path / "libfastvr_hostcheck.so")
    _build(lib, ["host_stubs.cpp", "host_stubs_rope_kv4.cpp"])
    driver = ("import sys, pytest\nfrom paper_2609_36757_amd import fastvr\nfastvr.LIB_PATH = sys.argv[1]\n"
              "sys.exit(pytest.main(['-q', '-p', 'no:cacheprovider', '-x', sys.argv[2]]))\n")
    assert " passed" in _run([driver, lib, os.path.join(ROOT, "tests", "test_abi_rope_kv4.py")])
    assert "valid calls done" in _run([VALID, lib, "0"])


def test_layer_without_kernels_refuses(tmp_path):
    lib = str(tmp_path / "libfastvr_nokernels.so")
    _build(lib, ["host_stubs.cpp"])
    assert "valid calls done" in _run([VALID, lib, "4"])
