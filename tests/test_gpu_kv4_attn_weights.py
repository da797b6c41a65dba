"""How exactly the attention over the 4-bit cache holds its softmax weights, on the GPU against the fp64 oracle.

Bound of an element of O, in parts of sum_j p_j |v_j|: a weight enters the products as a sum of two bf16 numbers, the
second one the rest of the first one's rounding, so it is off by half a step of half a step, 2^-8 2^-8; scores as in
kv4_checks.py; 2 n products are added in fp32, n + 64 sums of weights, 2^-24 each (64: the waves' and shares' joins); exp2 and the
products around it 2^-20.  A bf16 output is rounded once more."""
import math

import numpy as np
import pytest
import torch

from kv4_checks import make_cache
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


@pytest.mark.parametrize("case", [
    # B, Nq, H, Hkv, d, n, chunk_len, window, output type
    (1, 1, 12, 12, 128, 1000, None, -1, BF16),
    (1, 1, 2, 2, 128, 3, None, -1, FP32),
    (1, 1, 4, 1, 64, 9001, None, -1, FP32),
    (2, 37, 16, 4, 64, 5003, 1, -1, BF16),
    (2, 20, 4, 2, 128, 517, 1, 63, FP32),
    (1, 1200, 2, 1, 128, 1203, 1, -1, FP32),
    (1, 900, 8, 2, 64, 700, 48, 2, BF16),
    (1, 4300, 8, 1, 64, 4300, 1, -1, FP32),
    (1, 4300, 8, 1, 128, 4300, 1, -1, FP32),
], ids=lambda c: f"B{c[0]}q{c[1]}H{c[2]}of{c[3]}d{c[4]}n{c[5]}L{c[6]}W{c[7]}{str(c[8])[6:]}")
def test_weights_keep_more_than_bf16(dev, case):
    B, Nq, H, Hkv, d, n, L, W, ot = case
    print(f"\n[gpu case] kv4 weights {case}", flush=True)
    g = torch.Generator().manual_seed(n + Nq)
    q = torch.randn((B, Nq, H, d), generator=g).to(BF16)
    k, v = (torch.randn((B, n, Hkv, d), generator=g).to(BF16) for _ in range(2))
    cache, kk, vv = make_cache(fastvr, k, v, n + 3, 0xFF)
    o, _ = fastvr.kv4_attn(q.to(dev), fastvr.KV4Cache(*(t.to(dev) for t in cache)), n, chunk_len=L, window_chunks=W, out_dtype=ot)
    torch.cuda.synchronize()
    heads = sorted({0, H - 1})           # the oracle takes the first and the last query head
    pick = [h // (H // Hkv) for h in heads]
    scale = float(np.float32(1 / math.sqrt(d)))
    ref, _, spread, smax = kv4.attention(q[:, :, heads], kk[:, :, pick], vv[:, :, pick], [n] * B, chunk_len=L or n,
                                         window_chunks=W, scale=scale)
    score = (d + 1) * 2.0 ** -24 * smax.transpose(0, 2, 1)[..., None]
    tol = spread * (2.0 ** -16 + 2 * score + (3 * n + 64) * 2.0 ** -24 + 2.0 ** -20) + 1e-30
    if ot is BF16:
        tol = tol + 2.0 ** -8 * (np.abs(ref) + tol)
    worst = float((np.abs(o[:, :, heads].double().cpu().numpy() - ref) / tol).max())
    rel = float(np.linalg.norm(o[:, :, heads].double().cpu().numpy() - ref) / np.linalg.norm(ref))
    print(f"[parity] {case} {worst:.3f} of its bound, {rel:.2e} of the norm", flush=True)
    assert worst <= 1
