"""Helpers of the 4-bit cache's GPU tests: a cache of given values, and the comparison of an
attention's outputs with the fp64 oracle's.

Bounds: P is rounded to bf16 (half a step: 2^-8 of each) before P V, so an element of O is off by
at most 2^-8 sum_j p_j |v_j| ("spread"); scores are sums of d exact products in fp32, off by at
most (d + 1) 2^-24 of sum_c |q_c k_c| ("smax", times scale), and so, relatively, is each p, twice
with the sum below it; adding n keys in fp32 costs n 2^-24 of the spread at most, exp2 and the products
around it 2^-20; a bf16 output is rounded once more.  LSE: the score error, and the sum's and
logarithm's."""
import numpy as np
import torch

from oracle import kv4


def make_cache(fastvr, k, v, capacity, fill=0):
    """A cache (CPU tensors) of the oracle's codes for k/v [B, n, H, d], with every row behind them
    filled with `fill` bytes; and the values it stands for."""
    out, vals = [], []
    for x in (k, v):
        codes, scales = kv4.quantize(x)
        vals.append(kv4.values(codes, scales))
        B, n, H, d = x.shape
        for t in (kv4.pack(codes), scales):
            full = np.full((B, H, capacity, t.shape[-1]), fill, dtype=np.uint8)
            full[:, :, :n] = t.transpose(0, 2, 1, 3)
            out.append(torch.from_numpy(full))
    return fastvr.KV4Cache(*out), vals[0], vals[1]


def compare(o, lse, ref, n_keys, label):
    o_ref, lse_ref, spread, smax = ref
    d = o_ref.shape[-1]
    score = (d + 1) * 2.0 ** -24 * smax                                    # [B, H, Nq]
    per_row = (2.0 ** -8 + 2 * score + n_keys * 2.0 ** -24 + 2.0 ** -20).transpose(0, 2, 1)[..., None]
    tol = spread * per_row + 1e-30
    if o.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (np.abs(o_ref) + tol)
    got = o.double().cpu().numpy()
    err = np.abs(got - o_ref)
    assert np.isfinite(got).all(), label
    print(f"[parity] {label} O {float((err / tol).max()):.3f} of its bound", flush=True)
    assert (err <= tol).all(), (label, float((err / tol).max()))
    if lse is None:
        return
    got = lse.double().cpu().numpy()
    empty = np.isneginf(lse_ref)
    assert (np.isneginf(got) == empty).all(), label
    ltol = score + n_keys * 2.0 ** -24 + 2.0 ** -20 + 2.0 ** -21 * np.abs(np.where(empty, 0, lse_ref))
    lerr = np.abs(np.where(empty, 0, got) - np.where(empty, 0, lse_ref))
    assert (lerr <= ltol).all(), (label, float((lerr / ltol).max()))
