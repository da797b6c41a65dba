"""fp64 CPU oracle for the 4-bit KV cache and the attention over it.

TEST INFRASTRUCTURE ONLY: used by tests/; the HIP library never imports, links or
calls it.

The format (include/fastvr.h): magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign bit,
blocks of 32 elements along head_dim with one power-of-two scale.
"""
from __future__ import annotations

import numpy as np

from .one_step import _f64

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32


def quantize(x):
    """x [..., d] -> (codes [..., d] 0..15, scale bytes [..., d / 32]), by search: the scale is the
    one of the 251 with the largest magnitude in [3.5, 7) (the lowest for smaller, the highest for
    larger ones), a code the nearest magnitude, the even code of two equally near ones."""
    x = _f64(x)
    blocks = x.reshape(*x.shape[:-1], -1, BLOCK)
    a = np.abs(blocks).max(-1)
    bad = ~np.isfinite(a)
    a = np.where(bad, 0.0, a)
    edges = 3.5 * 2.0 ** np.arange(-124, 126)          # from edge i on: exponent i - 124
    e = np.searchsorted(edges, a, side="right") - 125
    y = np.abs(np.where(bad[..., None], 0.0, blocks)) / 2.0 ** e[..., None]
    off = np.abs(y[..., None] - MAGNITUDES)
    near = off == off.min(-1, keepdims=True)
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), near.argmax(-1))
    code = code + 8 * np.signbit(blocks)
    code = np.where(bad[..., None], 0, code)
    return code.reshape(x.shape).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def values(codes, scales) -> np.ndarray:
    """Codes [..., d] and scale bytes [..., d / 32] -> float64 [..., d]; byte 255 stands for NaN."""
    c = np.asarray(codes).astype(int)
    s = np.asarray(scales).astype(int)
    v = MAGNITUDES[c & 7] * np.where(c & 8, -1.0, 1.0)
    f = np.where(s == 255, np.nan, 2.0 ** (s - 127.0))
    return (v.reshape(*c.shape[:-1], -1, BLOCK) * f[..., None]).reshape(c.shape)


def pack(codes) -> np.ndarray:
    """[..., d] codes -> [..., d / 2] bytes, the even element in the low half."""
    return (codes[..., 0::2] | codes[..., 1::2] << 4).astype(np.uint8)


def unpack(packed) -> np.ndarray:
    p = np.asarray(packed)
    return np.stack((p & 15, p >> 4), -1).reshape(*p.shape[:-1], -1)


def visible(nq, length, chunk_len, window_chunks) -> np.ndarray:
    """[nq, length] truth values: which of `length` tokens the newest nq see."""
    pos = length - nq + np.arange(nq)
    diff = pos[:, None] // chunk_len - np.arange(length)[None] // chunk_len
    return (pos[:, None] >= 0) & (diff >= 0) & ((window_chunks < 0) | (diff <= window_chunks))


def attention(q, k, v, lens, *, chunk_len, window_chunks=-1, scale=1.0):
    """q [B, Nq, H, d], k/v [B, n, Hkv, d], lens [B] -> (O [B, Nq, H, d], LSE [B, H, Nq], spread, smax):
    spread = sum_j p_j |v_j| [B, Nq, H, d] and smax [B, H, Nq], the largest scale * sum_c |q_c k_c| of a
    visible key, are what rounding errors of P and of the scores are measured against."""
    q, k, v = _f64(q), _f64(k), _f64(v)
    B, Nq, H, d = q.shape
    G = H // k.shape[2]
    o, spread = np.zeros((B, Nq, H, d)), np.zeros((B, Nq, H, d))
    lse, smax = np.full((B, H, Nq), -np.inf), np.zeros((B, H, Nq))
    for b in range(B):
        n = int(lens[b])
        see = visible(Nq, n, chunk_len, window_chunks)
        for h in range(H):
            kk, vv = k[b, :n, h // G], v[b, :n, h // G]
            s = scale * (q[b, :, h] @ kk.T)
            size = abs(scale) * (np.abs(q[b, :, h]) @ np.abs(kk).T)
            for i in range(Nq):
                at = see[i]
                if not at.any():
                    continue
                m = s[i, at].max()
                w = np.exp(s[i, at] - m)
                lse[b, h, i] = m + np.log(w.sum())
                w /= w.sum()
                o[b, i, h] = w @ vv[at]
                spread[b, i, h] = w @ np.abs(vv[at])
                smax[b, h, i] = size[i, at].max()
    return o, lse, spread, smax
