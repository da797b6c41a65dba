"""kv4_read into K and V views that lie side by side in the rows of one buffer: of one token of
several sequences, whose rows are a batch stride apart, as of several tokens.  On the CPU against
stand-in launchers, under the sanitizers; on the GPU against separate outputs, bit for bit."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2609_36757_amd import fastvr
from test_host_sanitizers import pytestmark as needs_sanitizers
from test_host_sanitizers_rope_kv4 import ROOT, _build, _run

CALLS = """
import sys
from paper_2609_36757_amd import fastvr
fastvr.LIB_PATH = sys.argv[1]
import test_abi_rope_kv4 as t
HD = 2 * 128
def read(n, B, gap, st, sb, v_sb=None):
    kw = dict(n=n, B=B, k=t.KN, v=t.KN + 2 * gap, k_st=st, v_st=st, k_sb=sb, v_sb=sb if v_sb is None else v_sb)
    return fastvr.kv4_read_raw(*dict(t.COPY, **kw).values(), None)
OK, INV = fastvr.OK, fastvr.ERR_INVALID_ARGUMENT
for kw, want in ((dict(n=1, B=2, gap=HD, st=HD, sb=2 * HD), OK),            # strides as a [B, 1, 2 H, d] buffer's views give them
                 (dict(n=1, B=2, gap=HD, st=2 * HD, sb=2 * HD), OK),
                 (dict(n=1, B=5, gap=-HD, st=HD, sb=2 * HD), OK),           # V first
                 (dict(n=1, B=2, gap=3 * HD, st=HD, sb=4 * HD), OK),
                 (dict(n=2, B=2, gap=HD, st=2 * HD, sb=4 * HD), OK),
                 (dict(n=1, B=1, gap=HD, st=HD, sb=HD), OK),
                 (dict(n=1, B=2, gap=HD - 8, st=HD, sb=2 * HD), INV),       # K's end under V's start
                 (dict(n=1, B=2, gap=HD + 8, st=HD, sb=2 * HD), INV),       # V's end over the next sequence's K
                 (dict(n=1, B=3, gap=HD, st=HD, sb=2 * HD, v_sb=3 * HD), INV),
                 (dict(n=1, B=2, gap=0, st=HD, sb=2 * HD), INV),
                 (dict(n=2, B=2, gap=2 * HD, st=2 * HD, sb=8 * HD), INV)):  # V's first row is K's second
    got = read(**kw)
    assert got == want, (kw, got, fastvr.last_error())
print("reads done")
"""


@needs_sanitizers
def test_views_of_one_buffer_are_told_from_overlaps(tmp_path):
    lib = str(tmp_path / "libfastvr_hostcheck.so")
    _build(lib, ["host_stubs.cpp", "host_stubs_rope_kv4.cpp"])
    assert "reads done" in _run([CALLS, lib])


@pytest.mark.gpu
@pytest.mark.parametrize("B,n,d", [(1, 1, 128), (2, 1, 64), (16, 1, 128), (3, 2, 128)])
def test_read_into_one_buffer(B, n, d):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    print(f"\n[gpu case] kv4 read side by side B{B} n{n} d{d}", flush=True)
    H, cap = 3, 40
    g = torch.Generator().manual_seed(B)
    k, v = (torch.randn((B, cap, H, d), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    cache = fastvr.kv4_cache(B, cap, H, d)
    fastvr.kv4_append(cache, k, v)
    starts = (torch.arange(B, dtype=torch.int32) * 2 + 1).cuda()
    want_k, want_v = fastvr.kv4_read(cache, n, starts=starts)
    buf = torch.full((B, n, 2 * H + 1, d), 7.0, dtype=torch.bfloat16, device="cuda")
    fastvr.kv4_read(cache, n, starts=starts, k_out=buf[:, :, :H], v_out=buf[:, :, H:2 * H])
    torch.cuda.synchronize()
    assert torch.equal(buf[:, :, :H], want_k) and torch.equal(buf[:, :, H:2 * H], want_v) and (buf[:, :, 2 * H:] == 7).all()
