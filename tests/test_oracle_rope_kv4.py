"""Pins of the rotary and 4-bit cache oracles (CPU): closed forms, worked examples,
brute force and differences."""
import math

import numpy as np
import pytest
import torch

import oracle
from oracle import kv4, rope as orope
from paper_2609_36757_amd import fastvr


def test_rope_worked_example():
    x = np.zeros((1, 2, 1, 64))
    x[0, :, 0, :4] = [1.0, 2.0, 3.0, 4.0]
    f = [math.pi / 2, math.pi]
    y = orope.rope(x, np.array([0, 1]), f, layout="interleaved", amplitude=2.0)
    np.testing.assert_allclose(y[0, 0, 0, :4], [2, 4, 6, 8], atol=1e-15)
    # a quarter turn of (1, 2), half a turn of (3, 4)
    np.testing.assert_allclose(y[0, 1, 0, :4], [-4, 2, -6, -8], atol=1e-14)
    y = orope.rope(x, np.array([0, 1]), f, layout="half")
    # pairs (1, 3) and (2, 4)
    np.testing.assert_allclose(y[0, 1, 0, :4], [-3, -2, 1, -4], atol=1e-14)


@pytest.mark.parametrize("layout", ["interleaved", "half"])
def test_rope_scores_depend_on_distance_only(layout):
    g = np.random.default_rng(1)
    q, k = g.standard_normal((2, 1, 1, 1, 64))
    f, _ = fastvr.rope_inv_freq(24)
    dots = [float((orope.rope(q, [a], f, layout=layout) * orope.rope(k, [a - 7], f, layout=layout)).sum())
            for a in (0, 5, 1000)]
    np.testing.assert_allclose(dots, dots[0], atol=1e-11)


@pytest.mark.parametrize("layout", ["interleaved", "half"])
def test_rope_gradient_against_differences(layout):
    g = np.random.default_rng(2)
    x, dy = g.standard_normal((2, 1, 3, 2, 64))
    pos = g.integers(0, 50, (3, 3))
    f, _ = fastvr.rope_inv_freq(20, sections=(8, 6, 6))
    kw = dict(layout=layout, sections=(8, 6, 6), amplitude=1.3)
    dx = orope.rope(dy, pos, f, inverse=True, **kw)
    for at in [(0, 0, 0, 0), (0, 1, 1, 5), (0, 2, 0, 21), (0, 2, 1, 39), (0, 1, 0, 63)]:
        e = np.zeros_like(x)
        e[at] = 1e-5
        diff = ((orope.rope(x + e, pos, f, **kw) - orope.rope(x - e, pos, f, **kw)) * dy).sum() / 2e-5
        assert abs(diff - dx[at]) < 1e-8


def test_rope_inv_freq():
    f, a = fastvr.rope_inv_freq(64)
    assert a == 1.0 and f[0] == 1.0 and math.isclose(f[63], 10000 ** (-63 / 64))
    lin, _ = fastvr.rope_inv_freq(64, scaling="linear", factor=4.0)
    np.testing.assert_allclose(np.array(lin) * 4, f, rtol=1e-15)
    ntk, _ = fastvr.rope_inv_freq(64, scaling="ntk", factor=4.0)
    assert ntk[0] == 1.0 and math.isclose(ntk[63], f[63] / 4, rel_tol=1e-12)
    yarn, amp = fastvr.rope_inv_freq(64, scaling="yarn", factor=4.0, original_len=8192)
    assert math.isclose(amp, 1 + 0.1 * math.log(4))
    turns = [8192 * x / (2 * math.pi) for x in f]
    for x, y, t in zip(f, yarn, turns):
        assert y == x if t >= 32 else (math.isclose(y, x / 4) if t <= 1 else x / 4 < y < x)
    video, _ = fastvr.rope_inv_freq(64, sections=(22, 21, 21))
    assert video[0] == video[22] == video[43] == 1.0 and math.isclose(video[21], 10000 ** (-21 / 22))
    for bad in (dict(scaling="other"), dict(sections=(1, 2)), dict(scaling="yarn"), dict(base=0.0),
                dict(sections=(32, 32), scaling="ntk")):
        with pytest.raises(ValueError):
            fastvr.rope_inv_freq(64, **bad)


def test_quantize_worked_example():
    # largest 6.75 -> scale 1; ties to the even code; 7 halves the resolution
    x = np.zeros(64)
    x[:12] = [6.75, -0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.5, 0.2, 0.3, -0.0]
    x[32:36] = [7.0, 1.0, 0.5, -13.9]
    codes, scales = kv4.quantize(x)
    assert scales.tolist() == [127, 128]
    assert kv4.values(codes, scales)[:11].tolist() == [6, 0, 1, 1, 2, 2, 4, 4, -6, 0, 0.5]
    assert codes[1] == 8 and codes[11] == 8      # the sign of a zero stays
    assert kv4.values(codes, scales)[32:36].tolist() == [8, 1, 0, -12]
    assert kv4.unpack(kv4.pack(codes)).tolist() == codes.tolist()


def test_quantize_range_and_specials():
    for a, byte in [(0.0, 2), (2.0 ** -140, 2), (3.4 * 2.0 ** -124, 2), (3.5 * 2.0 ** -124, 3), (3.5, 127), (3.49, 126),
                    (6.99, 127), (3.3e38, 252), (np.inf, 255), (np.nan, 255)]:
        x = np.zeros(32)
        x[7] = a
        codes, scales = kv4.quantize(x)
        assert scales.tolist() == [byte], a
        v = kv4.values(codes, scales)
        if byte == 255:
            assert np.isnan(v).all() and (codes == 0).all()
        else:
            assert np.isfinite(v).all() and (v == torch.tensor(v).bfloat16().double().numpy()).all()


def test_quantize_error_bound():
    """An element is off by at most half its step: 1/7 of the block's largest above 4, a
    quarter of the scale below 2."""
    x = torch.randn(500, 128, generator=torch.Generator().manual_seed(3)).bfloat16().double().numpy()
    codes, scales = kv4.quantize(x)
    step = np.repeat(2.0 ** (scales - 127.0), 32, -1)
    y = np.abs(x) / step
    assert (y < 7).all() and (y.reshape(500, 4, 32).max(-1) >= 3.5).all()
    half = np.where(y >= 4, 1.0, np.where(y >= 2, 0.5, 0.25))
    assert (np.abs(kv4.values(codes, scales) - x) <= half * step).all()


def test_attention_equals_the_chunk_oracle():
    """The same function as the bf16 attention's oracle where both are defined: a query
    chunk at the end of a cache of whole chunks."""
    g = np.random.default_rng(4)
    L, c, n_new, H, d = 12, 3, 7, 2, 64
    n = c * L + n_new
    q = g.standard_normal((1, n_new, H, d))
    k, v = g.standard_normal((2, 1, n, H, d))
    for W in (-1, 0, 1, 2, 5):
        o, lse, _, _ = kv4.attention(q, k, v, [n], chunk_len=L, window_chunks=W, scale=0.2)
        o2, lse2 = oracle.attention(q, k, v, chunk_len=L, q_chunk_offset=c, window_chunks=W, scale=0.2)
        np.testing.assert_allclose(o, o2, atol=1e-12)
        np.testing.assert_allclose(lse, lse2, atol=1e-12)


def test_attention_groups_lengths_and_empty_rows():
    g = np.random.default_rng(5)
    q = g.standard_normal((2, 3, 4, 64))
    k, v = g.standard_normal((2, 2, 5, 2, 64))
    o, lse, _, _ = kv4.attention(q, k, v, [5, 2], chunk_len=1, scale=0.3)
    # sequence 1 holds two tokens: the first of its three rows is padding
    assert (o[1, 0] == 0).all() and np.isneginf(lse[1, :, 0]).all()
    # token-causal: its second row sees key 0 only, through key head h // 2
    for h in range(4):
        np.testing.assert_allclose(o[1, 1, h], v[1, 0, h // 2])
        w = np.exp(0.3 * q[0, 1, h] @ k[0, :4, h // 2].T)
        np.testing.assert_allclose(o[0, 1, h], w @ v[0, :4, h // 2] / w.sum())
