"""fp64 CPU oracle for rotary positions.

TEST INFRASTRUCTURE ONLY: used by tests/; the HIP library never imports, links or
calls it.

Pair p of a token is a complex number that is multiplied by
amplitude * exp(i * position * inv_freq[p]); the gradient of that product is the
product with the conjugate.
"""
from __future__ import annotations

import numpy as np

from .one_step import _f64


def rope(x, positions, inv_freq, *, layout="interleaved", sections=None, amplitude=1.0, inverse=False) -> np.ndarray:
    """x [B, N, H, d], positions [N, A] or [B, N, A] (or without A for one axis), inv_freq [P]; float64."""
    x = _f64(x).copy()
    B, N, H, d = x.shape
    f = _f64(inv_freq)
    P = len(f)
    sections = (P,) if sections is None else tuple(sections)
    assert sum(sections) == P
    pos = _f64(positions)
    if len(sections) == 1 and (pos.ndim == 1 or pos.shape == (B, N)) and pos.shape != (N, 1):
        pos = pos[..., None]
    pos = np.broadcast_to(pos, (B, N, len(sections)))
    axis = np.concatenate([np.full(n, a, dtype=int) for a, n in enumerate(sections)]) if P else np.zeros(0, int)
    turn = amplitude * np.exp((-1j if inverse else 1j) * pos[:, :, axis] * f)[:, :, None]
    if layout == "interleaved":
        first, second = np.arange(P) * 2, np.arange(P) * 2 + 1
    else:
        first, second = np.arange(P), np.arange(P) + P
    z = (x[..., first] + 1j * x[..., second]) * turn
    x[..., first], x[..., second] = z.real, z.imag
    return x
