"""Attention over the 4-bit cache on the GPU at sizes that reach every pair of its kernels (tests/kv4_plan_cases.py):
parity with the fp64 oracle, and what blocks that are not numbers reach, where a workgroup has several row tiles."""
import math

import numpy as np
import pytest
import torch

from kv4_checks import compare, make_cache
from kv4_plan_cases import PARITY, VISIBILITY, name
from oracle import kv4
from paper_2609_36757_amd import fastvr

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fastvr.load()
    return torch.device("cuda:0")


@pytest.mark.parametrize("c", PARITY, ids=name)
def test_parity(dev, c):
    """Full lengths, and lengths on the device that leave shares and rows without keys; NaN behind every
    sequence.  Two key heads are made and repeated, the oracle takes the first and the last sequence and one
    query head of the first and the last key head."""
    print(f"\n[gpu case] kv4 plans, parity {name(c)}", flush=True)
    g = torch.Generator().manual_seed(c.n + c.Nq)
    made = min(c.Hkv, 2)
    k = torch.randn((1, c.n, made, c.d), generator=g)
    k[:, ::37] *= 8
    v = torch.randn((1, c.n, made, c.d), generator=g)
    small, kk, vv = make_cache(fastvr, k.to(BF16), v.to(BF16), c.n + 5, 0xFF)
    # key head h holds head h * made // Hkv of those: the first and the last differ
    of = [h * made // c.Hkv for h in range(c.Hkv)]
    full = [t[:, of].repeat(c.B, 1, 1, 1) for t in small]
    q = torch.randn((c.B, c.Nq, c.H, c.d), generator=g).to(BF16)
    scale = float(np.float32(1 / math.sqrt(c.d)))
    G = c.H // c.Hkv
    heads = sorted({G // 2, c.H - 1})
    pick = [of[h // G] for h in heads]
    for lens in ([c.n] * c.B, [c.n - (b * 37 + c.n // 3) % c.n for b in range(c.B)]):
        cache = [t.clone() for t in full]
        for t in cache:
            for b, x in enumerate(lens):
                t[b, :, x:] = 0xFF
        cache = fastvr.KV4Cache(*(t.to(dev) for t in cache))
        t = torch.tensor(lens, dtype=torch.int32, device=dev)
        for ot in (FP32, BF16):
            o, lse = fastvr.kv4_attn(q.to(dev), cache, c.n, lens=t, chunk_len=c.L, window_chunks=c.W, out_dtype=ot)
            torch.cuda.synchronize()
            if ot is FP32:
                first = o, lse
            for b in sorted({0, c.B - 1}):
                if ot is FP32:
                    ref = kv4.attention(q[b:b + 1, :, heads], kk[:, :, pick], vv[:, :, pick], lens[b:b + 1], chunk_len=c.L,
                                        window_chunks=c.W, scale=scale)
                    refs = {b: ref} if b == 0 else {**refs, b: ref}
                compare(o[b:b + 1, :, heads], lse[b:b + 1, heads], refs[b], c.n, f"{name(c)} {b} {lens[b]}")
        # equal calls, equal bits
        o, lse = fastvr.kv4_attn(q.to(dev), cache, c.n, lens=t, chunk_len=c.L, window_chunks=c.W, out_dtype=FP32)
        assert torch.equal(o, first[0]) and torch.equal(lse, first[1])


def _rows_that_see(c, key, dev):
    return torch.from_numpy(kv4.visible(c.Nq, c.n, c.L, c.W)[:, key]).to(dev)


@pytest.mark.parametrize("ot", [FP32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("c", VISIBILITY, ids=name)
def test_what_is_no_number_reaches_the_rows_that_see_it(dev, c, ot):
    """A V block that stands for NaN makes its 32 elements of the rows that see the key NaN, a K block all of them
    and their LSE; every other bit is as without them.  Keys are chosen in different row tiles of
    one workgroup, whose own tokens they are, near the first queries, the middle and the end; scale bytes that are
    no part of the format, behind what a row sees, do nothing to it."""
    print(f"\n[gpu case] kv4 plans, visibility {name(c)} {ot}", flush=True)
    g = torch.Generator(device=dev).manual_seed(c.n)
    k, v = (torch.randn((c.B, c.n, c.Hkv, c.d), generator=g, device=dev).to(BF16) for _ in range(2))
    q = torch.randn((c.B, c.Nq, c.H, c.d), generator=g, device=dev).to(BF16)
    clean = fastvr.kv4_cache(c.B, c.n, c.Hkv, c.d)
    fastvr.kv4_append(clean, k, v)
    call = dict(chunk_len=c.L, window_chunks=c.W, out_dtype=ot)
    o0, lse0 = fastvr.kv4_attn(q, clean, c.n, **call)
    assert torch.isfinite(o0).all() and torch.isfinite(lse0).all()
    G, blocks = c.H // c.Hkv, c.d // 32
    tokens = 16 * c.tiles // G                                  # of a workgroup's rows
    for first in (0, c.Nq // 2 // tokens * tokens, (c.Nq - 1) // tokens * tokens):
        cache = fastvr.KV4Cache(*(t.clone() for t in clean))
        nan_o, nan_lse = torch.zeros_like(o0, dtype=torch.bool), torch.zeros_like(lse0, dtype=torch.bool)
        at = lambda i: min(c.n - c.Nq + first + i * tokens // 8, c.n - 1)  # noqa: E731
        for b in range(c.B):
            for hk in range(c.Hkv):
                heads = slice(hk * G, (hk + 1) * G)
                if hk % 2 == 0:
                    for j in range(blocks):                     # block j: a key of another row tile
                        key = at((3 * j + hk + b) % 8)
                        cache.v_scales[b, hk, key, j] = 255
                        cache.v_codes[b, hk, key, 16 * j:16 * j + 16] = 0
                        nan_o[b, :, heads, 32 * j:32 * j + 32] |= _rows_that_see(c, key, dev)[:, None, None]
                else:
                    key = at((5 * hk + b) % 8)
                    cache.k_scales[b, hk, key, hk % blocks] = 255
                    cache.k_codes[b, hk, key, 16 * (hk % blocks):16 * (hk % blocks) + 16] = 0
                    see = _rows_that_see(c, key, dev)
                    nan_o[b, :, heads] |= see[:, None, None]
                    nan_lse[b, heads] |= see
        o, lse = fastvr.kv4_attn(q, cache, c.n, **call)
        torch.cuda.synchronize()
        assert nan_o.any() and not nan_o.all() and nan_lse.any() and not nan_lse.all()
        assert torch.equal(torch.isnan(o), nan_o) and torch.equal(torch.isnan(lse), nan_lse), (first, name(c))
        assert torch.equal(o[~nan_o], o0[~nan_o]) and torch.equal(lse[~nan_lse], lse0[~nan_lse]), (first, name(c))
    # any bytes at all in the keys from `key` on: the rows that see none of them keep their bits
    key = c.n - c.Nq // 2
    cache = fastvr.KV4Cache(*(t.clone() for t in clean))
    for t in cache:
        t[:, :, key:] = torch.randint(0, 256, t[:, :, key:].shape, generator=g, device=dev, dtype=torch.uint8)
    cache.v_scales[:, :, key] = 253
    cache.k_scales[:, :, key] = 254
    rows = ~torch.from_numpy(kv4.visible(c.Nq, c.n, c.L, c.W)[:, key:].any(1)).to(dev)
    o, lse = fastvr.kv4_attn(q, cache, c.n, **call)
    assert rows.any() and torch.equal(o[:, rows], o0[:, rows]) and torch.equal(lse[..., rows], lse0[..., rows])
