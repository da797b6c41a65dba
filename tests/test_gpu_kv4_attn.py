"""Attention over the 4-bit cache on the GPU against the fp64 oracle on the values that the cache
stands for (bounds: kv4_checks.py)."""
import math

import numpy as np
import pytest
import torch

from kv4_checks import compare, make_cache
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


def inputs(B, Nq, H, Hkv, d, n, cap, seed, fill=0xFF):
    """q, a cache whose rows behind n are all ones (NaN scales), and its values."""
    g = torch.Generator().manual_seed(seed)
    q = torch.randn((B, Nq, H, d), generator=g).to(BF16)
    k = torch.randn((B, n, Hkv, d), generator=g) + 0.5 * torch.randn((1, 1, Hkv, d), generator=g)
    k[:, ::37] *= 8
    v = torch.randn((B, n, Hkv, d), generator=g)
    cache, kv, vv = make_cache(fastvr, k.to(BF16), v.to(BF16), cap, fill)
    return q, cache, kv, vv


def run(dev, q, cache, n, **kw):
    o, lse = fastvr.kv4_attn(q.to(dev), fastvr.KV4Cache(*(t.to(dev) for t in cache)), n, **kw)
    torch.cuda.synchronize()
    return o, lse


CASES = [
    # B, Nq, H, Hkv, d, n, extra capacity, chunk_len, window, output type
    (1, 1, 1, 1, 128, 1, 0, None, -1, FP32),
    (1, 1, 1, 1, 64, 1, 3, None, -1, BF16),
    (2, 1, 2, 2, 128, 31, 0, None, -1, FP32),
    (1, 1, 3, 3, 64, 33, 2, None, -1, FP32),
    (1, 1, 12, 12, 128, 1000, 24, None, -1, BF16),
    (3, 1, 8, 2, 128, 517, 11, None, -1, FP32),
    (1, 1, 2, 2, 128, 9001, 0, None, -1, FP32),        # keys split over workgroups
    (1, 1, 4, 1, 64, 8191, 1, None, -1, BF16),
    (1, 16, 1, 1, 128, 300, 0, None, -1, FP32),        # one full tile
    (1, 17, 1, 1, 128, 300, 0, None, -1, FP32),        # two tiles of a workgroup
    (2, 5, 6, 2, 64, 129, 3, 1, -1, FP32),             # token-causal, grouped
    (1, 37, 4, 4, 128, 700, 4, 1, -1, BF16),
    (1, 40, 2, 2, 64, 2100, 0, 1, 63, FP32),           # sliding window of 64 tokens
    (1, 200, 2, 1, 128, 200, 0, 1, -1, FP32),          # token-causal over a whole sequence
    (1, 64, 2, 2, 128, 256, 0, 64, 1, FP32),           # the newest chunk and the one before
    (2, 100, 2, 2, 64, 333, 7, 48, 2, FP32),           # rows of several chunks, from within one
    (1, 130, 3, 3, 128, 1111, 0, 130, -1, BF16),
    (1, 3, 64, 8, 128, 4000, 0, 1, -1, FP32),
    (1, 1601, 4, 1, 64, 1601, 2, 1, -1, FP32),         # a hundred row tiles of one key head
    (2, 1100, 4, 2, 128, 1203, 0, 60, 3, BF16),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"B{c[0]}q{c[1]}H{c[2]}of{c[3]}d{c[4]}n{c[5]}L{c[7]}W{c[8]}")
def test_attn_parity(dev, case):
    B, Nq, H, Hkv, d, n, extra, L, W, ot = case
    print(f"\n[gpu case] kv4 attn {case}", flush=True)
    q, cache, k, v = inputs(B, Nq, H, Hkv, d, n, n + extra, n + Nq)
    o, lse = run(dev, q, cache, n, chunk_len=L, window_chunks=W, out_dtype=ot)
    scale = float(np.float32(1 / math.sqrt(d)))
    compare(o, lse, kv4.attention(q, k, v, [n] * B, chunk_len=L or n, window_chunks=W, scale=scale), n, str(case))
    o2, lse2 = run(dev, q, cache, n, chunk_len=L, window_chunks=W, out_dtype=ot)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("case", [
    # B, Nq, H, Hkv, d, n, chunk_len, window, output type, whether tiles are split
    (33, 1, 33, 33, 64, 1500, None, -1, FP32, True),
    (1, 2100, 8, 2, 128, 5003, None, -1, BF16, True),
    (1, 4300, 8, 1, 64, 4300, 700, 2, FP32, True),
    (2, 2200, 8, 1, 128, 2600, 1, -1, FP32, False),
    (1, 4300, 8, 1, 128, 4300, 1, -1, FP32, True),
], ids=lambda c: f"B{c[0]}q{c[1]}H{c[2]}of{c[3]}d{c[4]}n{c[5]}L{c[6]}W{c[7]}")
def test_more_tiles_than_fit_at_once(dev, case):
    """One workgroup for the keys of most row tiles, several for those of the last ones: full
    lengths, and lengths that leave some workgroups without keys.  Where key heads are many, three are made
    and repeated; the oracle takes the first and the last sequence and one query head of each of their key heads."""
    B, Nq, H, Hkv, d, n, L, W, ot, split = case
    print(f"\n[gpu case] kv4 attn, many tiles {case}", flush=True)
    ws = fastvr.kv4_attn_workspace(B, H, Hkv, Nq, d, n, L or n, W)
    assert (ws > 0) == split and ws < B * H * Nq * (4 * d + 8)          # fewer than the rows have partial results
    made = min(Hkv, 3)
    _, cache, k, v = inputs(1, 1, made, made, d, n, n + 3, n + Nq)
    cache = fastvr.KV4Cache(*(t.repeat(B, Hkv // made, 1, 1) for t in cache))
    q = torch.randn((B, Nq, H, d), generator=torch.Generator().manual_seed(Nq)).to(BF16)
    scale = float(np.float32(1 / math.sqrt(d)))
    heads = [hk * (H // Hkv) + hk * 5 % (H // Hkv) for hk in list(range(Hkv))[-made:]]
    for lens in ([n] * B, [n - (b * 37 + 900) % n for b in range(B)]):
        t = torch.tensor(lens, dtype=torch.int32, device=dev)
        o, lse = run(dev, q, cache, n, lens=t, chunk_len=L, window_chunks=W, out_dtype=ot)
        for b in sorted({0, B - 1}):
            ref = kv4.attention(q[b:b + 1, :, heads], k, v, lens[b:b + 1], chunk_len=L or n, window_chunks=W, scale=scale)
            compare(o[b:b + 1, :, heads], lse[b:b + 1, heads], ref, n, f"{case} {b} {lens[b]}")
        o2, lse2 = run(dev, q, cache, n, lens=t, chunk_len=L, window_chunks=W, out_dtype=ot)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("Nq,L,W", [(1, None, -1), (1, 1, 99), (6, 1, -1), (40, 16, 1)])
def test_lengths_on_the_device(dev, Nq, L, W):
    """Lengths from none to all, fewer than Nq, and outside 0 .. cache_len; rows that see nothing."""
    print(f"\n[gpu case] kv4 attn lens Nq{Nq} L{L}", flush=True)
    lens = [0, 1, 3, 39, 1500, 2000, 2001, -7]
    B, H, Hkv, d, n = len(lens), 4, 2, 128, 2000
    q, cache, k, v = inputs(B, Nq, H, Hkv, d, n, n + 5, 77)
    real = [min(max(x, 0), n) for x in lens]
    # rows behind each sequence hold NaN
    for t in cache:
        for b, x in enumerate(real):
            t[b, :, x:] = 0xFF
    t = torch.tensor(lens, dtype=torch.int32, device=dev)
    o, lse = run(dev, q, cache, n, lens=t, chunk_len=L, window_chunks=W, scale=0.1)
    ref = kv4.attention(q, k, v, real, chunk_len=L or n, window_chunks=W, scale=float(np.float32(0.1)))
    compare(o, lse, ref, n, f"lens Nq{Nq}")
    assert (o[0] == 0).all() and torch.isneginf(lse[0]).all() and torch.isneginf(lse[7]).all()


@pytest.mark.parametrize("d", [64, 128])
def test_non_finite_keys_reach_only_rows_that_see_them(dev, d):
    """Token-causal rows over a cache with NaN blocks: a K block spoils the rows that see the
    key, a V block its 32 elements of them."""
    print(f"\n[gpu case] kv4 attn NaN d{d}", flush=True)
    B, Nq, H, n = 1, 20, 2, 100
    g = torch.Generator().manual_seed(9)
    q = torch.randn((B, Nq, H, d), generator=g).to(BF16)
    k, v = (torch.randn((B, n, H, d), generator=g).to(BF16) for _ in range(2))
    k[0, 95, 0, 3] = float("inf")
    v[0, 90, 1, 40] = float("nan")
    v[0, 93, 1, 5] = float("-inf")
    cache, _, _ = make_cache(fastvr, k, v, n)
    o, lse = run(dev, q, cache, n, chunk_len=1)
    pos = torch.arange(n - Nq, n, device=dev)
    # keys of one 32-key step with those rows: 64 .. 95, 96 .. 99
    assert torch.equal(torch.isnan(lse[0, 0]), pos >= 95) and not torch.isnan(lse[0, 1]).any()
    assert torch.equal(torch.isnan(o[0, :, 0]), (pos >= 95)[:, None].expand(Nq, d))
    want = torch.zeros((Nq, d), dtype=torch.bool, device=dev)
    want[pos >= 90, 32:64] = True
    want[pos >= 93, 0:32] = True
    assert torch.equal(torch.isnan(o[0, :, 1]), want)
    # steps that every row sees whole
    v2 = v.clone()
    v2[0, 3, 0, 33] = float("nan")
    cache, _, _ = make_cache(fastvr, k, v2, n)
    o, _ = run(dev, q, cache, n, chunk_len=1)
    assert torch.isnan(o[0, :, 0, 32:64]).all() and not torch.isnan(o[0, pos < 95, 0, :32]).any()
    # a NaN query row
    q2 = q.clone()
    q2[0, 4, 1, 0] = float("nan")
    cache, _, _ = make_cache(fastvr, k.nan_to_num(0, 0, 0), v.nan_to_num(0, 0, 0), n)
    o, lse = run(dev, q2, cache, n)
    bad = torch.zeros((Nq, H), dtype=torch.bool, device=dev)
    bad[4, 1] = True
    assert torch.equal(torch.isnan(o[0]), bad[..., None].expand(Nq, H, d)) and torch.equal(torch.isnan(lse[0].t()), bad)


@pytest.mark.parametrize("scale", [0.0, -0.09, 3.0, 1e-30])
def test_scales(dev, scale):
    print(f"\n[gpu case] kv4 attn scale {scale}", flush=True)
    B, Nq, H, d, n = 1, 19, 2, 128, 700
    q, cache, k, v = inputs(B, Nq, H, H, d, n, n + 1, 5)
    for L in (None, 1):
        o, lse = run(dev, q, cache, n, scale=scale, chunk_len=L)
        compare(o, lse, kv4.attention(q, k, v, [n], chunk_len=L or n, scale=float(np.float32(scale))), n, f"scale {scale}")


def test_views_outputs_and_canaries(dev):
    """q as a view of a packed projection, outputs into views: everything beside them stays."""
    print("\n[gpu case] kv4 attn views", flush=True)
    B, Nq, H, Hkv, d, n = 2, 7, 4, 2, 64, 6000
    q, cache, k, v = inputs(B, Nq, H, Hkv, d, n, n, 21)
    pack = torch.zeros((B, Nq + 2, 3 * H, d), dtype=BF16)
    pack[:, 1:Nq + 1, H:2 * H] = q
    dc = fastvr.KV4Cache(*(t.to(dev) for t in cache))
    dp = pack.to(dev)
    need = fastvr.kv4_attn_workspace(B, H, Hkv, Nq, d, n, n)
    assert need > 0
    for ot in (FP32, BF16):
        buf = torch.full((B, Nq + 2, H + 2, d), 7.0, dtype=ot, device=dev)
        ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device=dev)
        lse = torch.full((B * H * Nq + 8,), 7.0, dtype=FP32, device=dev)
        o, l2 = fastvr.kv4_attn(dp[:, 1:Nq + 1, H:2 * H], dc, n, out=buf[:, 1:Nq + 1, 1:H + 1], workspace=ws[:need],
                                lse=lse[:B * H * Nq].view(B, H, Nq))
        torch.cuda.synchronize()
        compare(o, l2, kv4.attention(q, k, v, [n] * B, chunk_len=n, scale=float(np.float32(1 / 8))), n, f"views {ot}")
        o.fill_(7.0)
        assert (buf == 7).all() and (lse[B * H * Nq:] == 7).all() and (ws[need:] == 0xFF).all()


def test_lse_is_optional(dev):
    q, cache, _, _ = inputs(1, 1, 2, 2, 64, 50, 50, 3)
    o, lse = run(dev, q, cache, 50)
    o2, none = run(dev, q, cache, 50, return_lse=False)
    assert none is None and torch.equal(o, o2)


def test_attn_refusals(dev):
    B, Nq, H, Hkv, d, n = 1, 2, 4, 2, 64, 5000
    cache = fastvr.kv4_cache(B, n, Hkv, d, dev)
    q = torch.zeros((B, Nq, H, d), dtype=BF16, device=dev)
    for kw in [dict(lens=torch.zeros(2, dtype=torch.int32, device=dev)), dict(lens=torch.zeros(1, device=dev)),
               dict(out_dtype=torch.float16), dict(out=torch.zeros_like(q), out_dtype=FP32), dict(out=q[:, :1]),
               dict(lse=torch.zeros((B, H, 3), device=dev)), dict(workspace=torch.zeros(4, device=dev)),
               dict(workspace=torch.zeros(4, dtype=torch.uint8))]:
        with pytest.raises(ValueError):
            fastvr.kv4_attn(q, cache, n, **kw)
    for kw, text in [(dict(chunk_len=0), "chunk_len"), (dict(window_chunks=-2), "window_chunks"),
                     (dict(scale=float("inf")), "scale"), (dict(out=q), "overlaps"),
                     (dict(workspace=torch.zeros(64, dtype=torch.uint8, device=dev)), "workspace")]:
        with pytest.raises(fastvr.FastVRError, match=text):
            fastvr.kv4_attn(q, cache, n, **kw)
    for args in [(q.float(), cache, n), (q.cpu(), cache, n), (q[..., :32], cache, n), (q.repeat(2, 1, 1, 1), cache, n)]:
        with pytest.raises(ValueError):
            fastvr.kv4_attn(*args)
    with pytest.raises(fastvr.FastVRError, match="capacity"):
        fastvr.kv4_attn(q, cache, n + 1)
    with pytest.raises(fastvr.FastVRError, match="multiple"):
        fastvr.kv4_attn(q[:, :, :3], cache, n)
    o, lse = fastvr.kv4_attn(q, cache, 0)
    assert (o == 0).all() and torch.isneginf(lse).all()
    assert fastvr.kv4_attn(q[:, :0], cache, n)[0].shape == (B, 0, H, d)


def test_rows_do_not_depend_on_keys_they_do_not_see(dev):
    """Token-causal rows that share tiles and steps: other keys behind a row, of any size, leave its
    bits as they were."""
    print("\n[gpu case] kv4 attn, keys behind a row", flush=True)
    B, Nq, H, d, n = 1, 48, 2, 128, 500
    q, cache, _, _ = inputs(B, Nq, H, H, d, n, n, 31)
    o, lse = run(dev, q, cache, n, chunk_len=1)
    other = [t.clone() for t in cache]
    g = torch.Generator().manual_seed(32)
    first = n - Nq // 2           # keys from here on change: larger, of both signs, one NaN
    for i in (0, 2):
        other[i][:, :, first:] = torch.randint(0, 256, other[i][:, :, first:].shape, generator=g, dtype=torch.uint8)
        other[i + 1][:, :, first:] = 131
    other[3][:, 0, n - 1, 1] = 255
    o2, lse2 = run(dev, q, other, n, chunk_len=1)
    same = first - (n - Nq)       # rows before the first changed key
    assert torch.equal(o[:, :same], o2[:, :same]) and torch.equal(lse[..., :same], lse2[..., :same])
    assert not torch.equal(o[:, same:], o2[:, same:])
