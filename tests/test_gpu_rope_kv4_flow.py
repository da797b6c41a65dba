"""Rotary positions, the 4-bit cache and its attention together, as a model's layer uses them:
a stream of chunks, single tokens of a ragged batch (eager and as a replayed graph), a ring of chunk
slots, two streams at once, and training's gradients; and caches and tensors past 2^31 bytes.

The oracle's attention takes the values that the cache's bytes stand for; that those are the quantised
rotated keys is asserted on its own."""
import math

import numpy as np
import pytest
import torch

import oracle
from kv4_checks import compare
from oracle import kv4, rope as orope
from paper_2609_36757_amd import fastvr

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fastvr.load()
    return torch.device("cuda:0")


def values(cache, n):
    """fp64 keys and values [B, n, H, d] of the first n rows, from the cache's bytes on the host."""
    out = []
    for codes, scales in ((cache[0], cache[1]), (cache[2], cache[3])):
        v = kv4.values(kv4.unpack(codes[:, :, :n].cpu().numpy()), scales[:, :, :n].cpu().numpy())
        out.append(np.ascontiguousarray(v.transpose(0, 2, 1, 3)))
    return out


def projections(B, N, H, d, dev, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((B, N, 3 * H, d), generator=g).to(BF16).to(dev)


def test_streamed_chunks(dev):
    """Chunks of a video stream: q and k turn in place in the packed projection, k and v go to the
    cache, q attends to it; W = 1 and unbounded windows."""
    print("\n[gpu case] flow, streamed chunks", flush=True)
    B, H, d, L, chunks, P = 1, 3, 128, 60, 4, 64
    qkv = projections(B, L * chunks - 17, H, d, dev, 1)
    N = qkv.shape[1]
    sections = (22, 21, 21)
    f = torch.tensor(fastvr.rope_inv_freq(P, sections=sections)[0], dtype=torch.float64, device=dev)
    i = torch.arange(N)
    pos = torch.stack((i // 30, i // 6 % 5, i % 6), 1).to(torch.int32).to(dev)
    raw = qkv.clone()
    for W in (-1, 1):
        cache, n = fastvr.kv4_cache(B, N + 3, H, d, dev), 0
        work = raw.clone()
        for c in range(chunks):
            s = slice(c * L, min((c + 1) * L, N))
            x = work[:, s]
            fastvr.rope(x[:, :, :2 * H], pos[s].contiguous(), f, sections=sections, out=x[:, :, :2 * H])
            n = fastvr.kv4_append(cache, x[:, :, H:2 * H], x[:, :, 2 * H:], n)
            o, lse = fastvr.kv4_attn(x[:, :, :H], cache, n, chunk_len=L, window_chunks=W)
            torch.cuda.synchronize()
            k, v = values(cache, n)
            ref = kv4.attention(x[:, :, :H], k, v, [n], chunk_len=L, window_chunks=W, scale=float(np.float32(1 / math.sqrt(d))))
            compare(o, lse, ref, n, f"chunk {c} W {W}")
        assert n == N
        turned = orope.rope(raw[:, :, :2 * H], pos.cpu(), f, sections=sections)
        assert np.abs(work[:, :, :2 * H].double().cpu().numpy() - turned).max() <= 2.0 ** -8 * np.abs(turned).max() + 1e-5
        assert torch.equal(work[:, :, 2 * H:], raw[:, :, 2 * H:])
        want = kv4.values(*kv4.quantize(work[:, :, H:2 * H]))
        np.testing.assert_array_equal(values(cache, N)[0], want)


def test_ring_of_chunk_slots(dev):
    """A ring of W + 1 slots: the newest chunk overwrites the oldest, and its queries see every
    row; the same as attention over the last chunks in order, up to the order of the sums."""
    print("\n[gpu case] flow, ring", flush=True)
    B, H, d, L, W = 1, 2, 64, 40, 1
    qkv = projections(B, 5 * L, H, d, dev, 2)
    ring, full = fastvr.kv4_cache(B, (W + 1) * L, H, d, dev), fastvr.kv4_cache(B, 5 * L, H, d, dev)
    for c in range(5):
        x = qkv[:, c * L:(c + 1) * L]
        fastvr.kv4_append(ring, x[:, :, H:2 * H], x[:, :, 2 * H:], c % (W + 1) * L)
        n = fastvr.kv4_append(full, x[:, :, H:2 * H], x[:, :, 2 * H:], c * L)
        held = min(n, (W + 1) * L)
        o, lse = fastvr.kv4_attn(x[:, :, :H], ring, held)
        torch.cuda.synchronize()
        k, v = values(full, n)
        ref = kv4.attention(x[:, :, :H], k, v, [n], chunk_len=L, window_chunks=W, scale=0.125)
        compare(o, lse, ref, n, f"ring chunk {c}")


def _tokens(t):
    """One decoding step of a ragged batch on the current stream, everything in t's buffers."""
    H, Hkv = t["H"], t["Hkv"]
    fastvr.rope(t["x"][:, :, :H + Hkv], t["pos"], t["f"], layout="half", out=t["qk"])
    fastvr.kv4_append(t["cache"], t["qk"][:, :, H:], t["x"][:, :, H + Hkv:], starts=t["lens"])
    t["lens"].add_(1)
    t["pos"].add_(1)
    fastvr.kv4_attn(t["qk"][:, :, :H], t["cache"], t["cap"], lens=t["lens"], out=t["o"], lse=t["lse"], workspace=t["ws"])


def test_tokens_eager_and_replayed(dev):
    """Token after token of a ragged batch, lengths on the device: a captured step, replayed with eager
    work in between, gives the eager steps' results bit for bit, and those are the oracle's."""
    print("\n[gpu case] flow, tokens", flush=True)
    B, H, Hkv, d, cap = 4, 8, 2, 128, 1500
    g = torch.Generator().manual_seed(3)
    start = [0, 700, 33, 1490]
    steps = 6
    xs = torch.randn((steps, B, 1, H + 2 * Hkv, d), generator=g).to(BF16).to(dev)
    old = torch.randn((2, B, cap, Hkv, d), generator=g).to(BF16).to(dev)

    def fresh():
        t = dict(H=H, Hkv=Hkv, cap=cap, x=xs[0].clone(), cache=fastvr.kv4_cache(B, cap, Hkv, d, dev))
        fastvr.kv4_append(t["cache"], old[0], old[1], 0)
        t["lens"] = torch.tensor(start, dtype=torch.int32, device=dev)
        t["pos"] = t["lens"].clone().view(B, 1)
        t["f"] = torch.tensor(fastvr.rope_inv_freq(32)[0], dtype=torch.float64, device=dev)
        t["qk"] = torch.empty((B, 1, H + Hkv, d), dtype=BF16, device=dev)
        t["o"] = torch.empty((B, 1, H, d), dtype=BF16, device=dev)
        t["lse"] = torch.empty((B, H, 1), dtype=FP32, device=dev)
        t["ws"] = torch.empty(max(1, fastvr.kv4_attn_workspace(B, H, Hkv, 1, d, cap, cap)), dtype=torch.uint8, device=dev)
        return t

    t = fresh()
    eager = []
    for i in range(steps):
        t["x"].copy_(xs[i])
        _tokens(t)
        torch.cuda.synchronize()
        lens = [s + i + 1 for s in start]
        k, v = values(t["cache"], cap)
        compare(t["o"], t["lse"], kv4.attention(t["qk"][:, :, :H], k, v, lens, chunk_len=cap,
                                                scale=float(np.float32(1 / math.sqrt(d)))), cap, f"token {i}")
        eager.append((t["o"].clone(), t["lse"].clone(), t["qk"].clone(), [c.clone() for c in t["cache"]]))

    t = fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _tokens(t)                      # eager once, on a stream of its own
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _tokens(t)
    for name in ("lens", "pos"):        # back to the start; the first step's rows are written again
        t[name].sub_(1)
    torch.cuda.synchronize()
    for i in range(steps):
        t["x"].copy_(xs[i])
        t["o"].fill_(float("nan"))
        t["ws"].fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        junk = torch.randn(1000, device=dev).sum()   # the program's own work
        torch.cuda.synchronize()
        o, lse, qk, cache = eager[i]
        assert torch.equal(t["o"], o) and torch.equal(t["lse"], lse) and torch.equal(t["qk"], qk), i
        assert all(torch.equal(a, b) for a, b in zip(t["cache"], cache)), i
        assert torch.isfinite(junk)


def test_two_streams_at_once(dev):
    """Two layers' calls on two streams, each with a workspace, against the same calls one by one."""
    print("\n[gpu case] flow, two streams", flush=True)
    B, H, d, n = 2, 4, 128, 6000
    sets = []
    for seed in (4, 5):
        kv = projections(B, n, 1, d, dev, seed).view(B, n, 3, d)
        kv = kv.repeat_interleave(H, 2)
        cache = fastvr.kv4_cache(B, n, H, d, dev)
        fastvr.kv4_append(cache, kv[:, :, H:2 * H], kv[:, :, 2 * H:], 0)
        sets.append((kv[:, :1, :H].contiguous(), cache))
    torch.cuda.synchronize()
    alone = [[x.clone() for x in fastvr.kv4_attn(q, c, n)] for q, c in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for rep in range(20):
        got = []
        for s, (q, c) in zip(streams, sets):
            with torch.cuda.stream(s):
                got.append(fastvr.kv4_attn(q, c, n))
        torch.cuda.synchronize()
        for a, b in zip(alone, got):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]), rep


def test_stream_argument(dev):
    """The stream= argument of each call orders its work on that stream."""
    print("\n[gpu case] flow, stream argument", flush=True)
    s = torch.cuda.Stream()
    B, H, d, n = 1, 2, 64, 300
    qkv = projections(B, n, H, d, dev, 6)
    f = torch.tensor(fastvr.rope_inv_freq(32)[0], dtype=torch.float64, device=dev)
    pos = torch.arange(n, dtype=torch.int32, device=dev)
    want = fastvr.rope(qkv, pos, f)
    cache = fastvr.kv4_cache(B, n, H, d, dev)
    out, lse = torch.empty((B, n, H, d), device=dev), torch.empty((B, H, n), device=dev)
    ws = torch.empty(max(1, fastvr.kv4_attn_workspace(B, H, H, n, d, n, n)), dtype=torch.uint8, device=dev)
    turned, ko, vo = torch.empty_like(qkv), *(torch.empty((B, n, H, d), dtype=BF16, device=dev) for _ in range(2))
    torch.cuda.synchronize()
    fastvr.rope(qkv, pos, f, out=turned, stream=s)
    fastvr.kv4_append(cache, turned[:, :, H:2 * H], turned[:, :, 2 * H:], 0, stream=s)
    fastvr.kv4_read(cache, n, k_out=ko, v_out=vo, stream=s)
    fastvr.kv4_attn(turned[:, :, :H], cache, n, out=out, lse=lse, workspace=ws, stream=s)
    s.synchronize()
    assert torch.equal(turned, want)
    k, v = values(cache, n)
    assert np.array_equal(ko.double().cpu().numpy(), k) and np.array_equal(vo.double().cpu().numpy(), v)
    compare(out, lse, kv4.attention(turned[:, :, :H], k, v, [n], chunk_len=n, scale=0.125), n, "stream argument")


def test_stream_argument_allocates_there(dev):
    """What a call on another stream allocates by itself, its workspace too, is that stream's memory: tensors
    made and filled on the current stream while the call still waits for its turn take none of it."""
    print("\n[gpu case] flow, allocations of another stream", flush=True)
    s = torch.cuda.Stream()
    B, H, d, n = 2, 12, 128, 4000
    k, v = (projections(B, n, H, d, dev, seed)[:, :, :H] for seed in (8, 9))
    q = projections(B, 1, H, d, dev, 10)[:, :, :H]
    f = torch.tensor(fastvr.rope_inv_freq(64)[0], dtype=torch.float64, device=dev)
    pos = torch.arange(n, dtype=torch.int32, device=dev)
    cache = fastvr.kv4_cache(B, n, H, d, dev)
    fastvr.kv4_append(cache, k, v)
    n_ws = fastvr.kv4_attn_workspace(B, H, H, 1, d, n, n)
    assert n_ws > 0
    want = (*fastvr.kv4_attn(q, cache, n), fastvr.rope(k, pos, f), *fastvr.kv4_read(cache, n))
    work = torch.randn((8192, 8192), device=dev)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(4):
            work = work @ work                    # some 10 ms ahead of the calls
    got = (*fastvr.kv4_attn(q, cache, n, stream=s), fastvr.rope(k, pos, f, stream=s),
           *fastvr.kv4_read(cache, n, stream=s))
    junk = [torch.full((max(1, size // 4),), float("nan"), device=dev)
            for size in (n_ws, *(t.numel() * t.element_size() for t in got)) for _ in range(2)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert all(bool(t.isnan().all()) for t in junk)

    class Elsewhere:
        cuda_stream, device_index = 0, 1
    for call in (lambda: fastvr.kv4_attn(q, cache, n, stream=Elsewhere), lambda: fastvr.rope(k, pos, f, stream=Elsewhere),
                 lambda: fastvr.kv4_append(cache, k, v, stream=Elsewhere)):
        with pytest.raises(ValueError, match="the stream is on cuda:1"):
            call()


def test_training_gradients(dev):
    """Loss gradients through rotary positions and the chunk attention: rope -> chunk_attn ->
    chunk_attn_bwd -> rope_bwd against the oracles' chain in fp64.  The attention's gradients differ from
    theirs by bf16 roundings of P and dS (the bar of the attention's own tests); turning adds 1e-6."""
    print("\n[gpu case] flow, training", flush=True)
    B, N, H, d, L, P = 1, 210, 2, 64, 70, 24
    g = torch.Generator().manual_seed(7)
    q, k, v, do = (torch.randn((B, N, H, d), generator=g).to(BF16).to(dev) for _ in range(4))
    f, amp = fastvr.rope_inv_freq(P, scaling="yarn", factor=4.0, original_len=64)
    ft = torch.tensor(f, dtype=torch.float64, device=dev)
    pos = torch.arange(100, 100 + N, dtype=torch.int32, device=dev)
    kw = dict(layout="half", amplitude=amp)
    qr, kr = fastvr.rope(q, pos, ft, **kw), fastvr.rope(k, pos, ft, **kw)
    o, lse = fastvr.chunk_attn(qr, kr, v, chunk_len=L, window_chunks=1)
    dq, dk, dv = fastvr.chunk_attn_bwd(qr, kr, v, o, lse, do, chunk_len=L, window_chunks=1)
    dq_raw = dq.clone()
    dx_q = fastvr.rope_bwd(dq, pos, ft, out=dq, **kw)       # in place, fp32
    dx_k = fastvr.rope_bwd(dk, pos, ft, **kw)
    torch.cuda.synchronize()
    assert dx_q.data_ptr() == dq.data_ptr() and not torch.equal(dq, dq_raw)
    scale = float(np.float32(1 / math.sqrt(d)))
    rq, rk, rv = oracle.attention_bwd(qr.cpu(), kr.cpu(), v.cpu(), do.cpu(), chunk_len=L, window_chunks=1, scale=scale)
    for got, ref in ((dx_q, orope.rope(rq, pos.cpu(), f, inverse=True, **kw)),
                     (dx_k, orope.rope(rk, pos.cpu(), f, inverse=True, **kw)), (dv, rv)):
        rel = np.linalg.norm(got.double().cpu().numpy() - ref) / np.linalg.norm(ref)
        assert rel <= 1e-2, rel
    # and the turning itself, of the very gradients that went in
    ref = orope.rope(dq_raw, pos.cpu(), f, inverse=True, **kw)
    assert np.abs(dx_q.double().cpu().numpy() - ref).max() <= 4e-6 * float(dq_raw.abs().max())


def test_cache_past_two_gigabytes(dev):
    """A cache of the largest capacity (16 Mi rows a head, 2 GB of codes for K and for V): rows at its end,
    written by starts, and keys in between that are zero, so that the sums are known."""
    print("\n[gpu case] flow, largest capacity", flush=True)
    H, d, cap, m = 2, 128, 16 * 1024 * 1024, 40
    cache = fastvr.kv4_cache(1, cap, H, d, dev)
    g = torch.Generator().manual_seed(8)
    k, v, q = (torch.randn((1, m, H, d), generator=g).to(BF16) for _ in range(3))
    st = torch.tensor([cap - m], dtype=torch.int32, device=dev)
    fastvr.kv4_append(cache, k.to(dev), v.to(dev), starts=st)
    ko, vo = fastvr.kv4_read(cache, m, cap - m)
    torch.cuda.synchronize()
    kv, vv = kv4.values(*kv4.quantize(k)), kv4.values(*kv4.quantize(v))
    assert np.array_equal(ko.double().cpu().numpy(), kv) and np.array_equal(vo.double().cpu().numpy(), vv)
    assert int(cache.v_codes[:, :, :cap - m].count_nonzero()) == 0
    o, lse = fastvr.kv4_attn(q[:, :2].to(dev), cache, cap, scale=0.7)
    ow, lw = fastvr.kv4_attn(q[:, :2].to(dev), cache, cap, scale=0.7, chunk_len=1, window_chunks=m // 2)
    torch.cuda.synchronize()
    # zero keys: score 0 each; enough weight on the last rows that they show (scale 0.7: scores of +-25)
    for h in range(H):
        s = float(np.float32(0.7)) * (q[0, :2, h].double().numpy() @ kv[0, :, h].T)
        top = np.maximum(s.max(1, keepdims=True), 0)
        z = np.exp(s - top).sum(1) + (cap - m) * np.exp(-top[:, 0])
        ref = (np.exp(s - top) @ vv[0, :, h]) / z[:, None]
        spread = (np.exp(s - top) @ np.abs(vv[0, :, h])) / z[:, None]
        size = float(np.float32(0.7)) * (np.abs(q[0, :2, h].double().numpy()) @ np.abs(kv[0, :, h]).T).max(1)
        # P to bf16, the scores' and the sum's fp32 additions (16 lanes add cap / (16 splits) keys each)
        tol = 2.0 ** -8 + 2 * 129 * 2.0 ** -24 * size + 2.0 ** -20 + cap / 256 * 2.0 ** -24
        assert (np.abs(o[0, :, h].double().cpu().numpy() - ref) <= spread * tol[:, None] + 1e-12).all()
        assert (np.abs(lse[0, h].double().cpu().numpy() - (top[:, 0] + np.log(z))) <= tol).all()
    ref = kv4.attention(q[:, :2], kv, vv, [m], chunk_len=1, window_chunks=m // 2, scale=float(np.float32(0.7)))
    compare(ow, lw, ref, m, "window at the end of the largest cache")


def test_rope_past_two_gigaelements(dev):
    """x of 2.2 G elements (4.4 GB), in place: the last tokens against the oracle, the first too."""
    print("\n[gpu case] flow, rope of 2.2 G elements", flush=True)
    N, H, d = 1_440_000, 12, 128
    x = torch.zeros((1, N, H, d), dtype=BF16, device=dev)
    g = torch.Generator().manual_seed(9)
    ends = torch.randn((2, 3, H, d), generator=g).to(BF16)
    x[0, :3], x[0, -3:] = ends[0].to(dev), ends[1].to(dev)
    f, _ = fastvr.rope_inv_freq(64)
    pos = torch.arange(N, dtype=torch.int32, device=dev)
    fastvr.rope(x, pos, torch.tensor(f, dtype=torch.float64, device=dev), out=x)
    torch.cuda.synchronize()
    for got, raw, p in ((x[:, :3], ends[:1], pos[:3]), (x[:, -3:], ends[1:], pos[-3:])):
        ref = orope.rope(raw, p.cpu(), f)
        assert (np.abs(got.double().cpu().numpy() - ref) <= 2.0 ** -8 * np.abs(ref) + 2e-5).all()
    assert int(x[0, 3:-3].count_nonzero()) == 0
