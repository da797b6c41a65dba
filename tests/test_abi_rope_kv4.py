"""C-ABI checks of the rotary and 4-bit cache entry points that need no GPU: every case is
rejected on the host before the HIP runtime is touched, so the device addresses are made up."""
import ctypes

import pytest

from paper_2609_36757_amd import fastvr

# Distinct made-up addresses, 1 TiB apart.
X, Y, POS, FREQ, KC, KS, VC, VS, KN, VN, ST, Q, O, LSE, WS, LENS = ((i + 1) << 40 for i in range(16))
INV, UNS, CAP = fastvr.ERR_INVALID_ARGUMENT, fastvr.ERR_UNSUPPORTED, fastvr.ERR_CAPACITY
BIG = 1 << 62

ROPE = dict(x=X, x_sb=16 * 256, x_st=256, x_fp32=0, y=Y, y_sb=16 * 256, y_st=256, y_fp32=0, positions=POS, pos_sb=0, n_axes=1,
            split1=32, split2=32, inv_freq=FREQ, n_pairs=32, amplitude=1.0, interleaved=1, inverse=0, B=2, N=16, H=2, d=128)
COPY = dict(k_codes=KC, k_scales=KS, v_codes=VC, v_scales=VS, k=KN, k_sb=3 * 256, k_st=256, v=VN, v_sb=3 * 256, v_st=256,
            starts=None, B=2, H=2, d=128, capacity=64, first=10, n=3)
ATTN = dict(q=Q, q_sb=2 * 512, q_st=512, k_codes=KC, k_scales=KS, v_codes=VC, v_scales=VS, o=O, o_sb=2 * 512, o_st=512, o_bf16=0,
            lse=LSE, workspace=WS, workspace_bytes=1 << 30, lens=None, B=2, H=4, Hkv=2, Nq=2, d=128, capacity=9000,
            cache_len=9000, chunk_len=9000, window_chunks=-1, scale=0.1)


def _refused(raw, good, kw, status, needle):
    args = dict(good, **kw)
    assert raw(*args.values(), None) == status, fastvr.last_error()
    assert needle in fastvr.last_error()


@pytest.fixture(scope="module", autouse=True)
def lib():
    return fastvr.load()


@pytest.mark.parametrize("kw,status,needle", [
    (dict(x=None), INV, "x is NULL"), (dict(y=None), INV, "y is NULL"), (dict(positions=None), INV, "positions is NULL"),
    (dict(inv_freq=None), INV, "inv_freq is NULL"), (dict(x=X + 8), INV, "aligned"), (dict(positions=POS + 2), INV, "aligned"),
    (dict(inv_freq=FREQ + 4), INV, "aligned"), (dict(B=-1), INV, "negative"), (dict(N=-1), INV, "negative"),
    (dict(H=-2), INV, "negative"), (dict(d=96), UNS, "head_dim"), (dict(x_fp32=2), INV, "x_fp32"), (dict(y_fp32=-1), INV, "y_fp32"),
    (dict(interleaved=2), INV, "interleaved"), (dict(inverse=3), INV, "inverse"), (dict(n_pairs=65, split1=65, split2=65), INV, "n_pairs"),
    (dict(n_pairs=-1), INV, "n_pairs"), (dict(n_axes=0), INV, "n_axes"), (dict(n_axes=4), INV, "n_axes"),
    (dict(split1=31), INV, "axes"), (dict(n_axes=2, split1=10, split2=31), INV, "axes"), (dict(n_axes=3, split1=10, split2=9), INV, "axes"),
    (dict(n_axes=3, split1=10, split2=33), INV, "axes"), (dict(n_axes=3, split1=-1), INV, "axes"),
    (dict(amplitude=float("nan")), INV, "amplitude"), (dict(amplitude=1e300), INV, "amplitude"),
    (dict(x_st=128), INV, "token stride"), (dict(y_st=260), INV, "multiples"), (dict(x_sb=256), INV, "batch stride"),
    (dict(pos_sb=15), INV, "positions batch stride"), (dict(pos_sb=-16), INV, "positions batch stride"),
    (dict(B=65536), UNS, "B > 65535"), (dict(N=(1 << 24) + 1), UNS, "2^24"), (dict(H=65536), UNS, "H > 65535"),
    (dict(y=X + 256), INV, "y overlaps x"), (dict(y=X, y_fp32=1), INV, "y overlaps x"), (dict(y=X, y_st=512, y_sb=16 * 512), INV, "overlaps x"),
    (dict(y=POS), INV, "positions"), (dict(y=FREQ), INV, "inv_freq"), (dict(x_sb=BIG, B=3), INV, "overflow"),
])
def test_rope_refuses(kw, status, needle):
    _refused(fastvr.rope_raw, ROPE, kw, status, needle)


@pytest.mark.parametrize("kw", [dict(B=0), dict(N=0), dict(H=0), dict(B=0, x=None, y=None, positions=None, inv_freq=None)])
def test_rope_empty(kw):
    assert fastvr.rope_raw(*dict(ROPE, **kw).values(), None) == fastvr.OK and fastvr.last_error() == ""


@pytest.mark.parametrize("raw", [fastvr.kv4_append_raw, fastvr.kv4_read_raw], ids=["append", "read"])
@pytest.mark.parametrize("kw,status,needle", [
    (dict(k_codes=None), INV, "k_codes is NULL"), (dict(k_scales=None), INV, "k_scales is NULL"), (dict(v_codes=None), INV, "v_codes is NULL"),
    (dict(v_scales=None), INV, "v_scales is NULL"), (dict(k=None), INV, "is NULL"), (dict(v=None), INV, "is NULL"),
    (dict(k_codes=KC + 8), INV, "aligned"), (dict(v_scales=VS + 4), INV, "aligned"), (dict(k=KN + 2), INV, "aligned"),
    (dict(starts=ST + 2), INV, "starts"), (dict(d=32), UNS, "head_dim"), (dict(B=-1), INV, "negative"), (dict(n=-1), INV, "negative"),
    (dict(capacity=-1), INV, "negative"), (dict(first=-1), INV, "first"), (dict(first=62), CAP, "capacity"),
    (dict(first=BIG, n=BIG), CAP, "capacity"), (dict(capacity=(1 << 24) + 1), UNS, "capacity"), (dict(B=32768), UNS, "32767"),
    (dict(H=65536), UNS, "65535"), (dict(k_st=128), INV, "token stride"), (dict(v_sb=256), INV, "batch stride"), (dict(v_st=258), INV, "multiples"),
    (dict(k=KC + 1024), INV, "overlaps"), (dict(v=VS), INV, "overlaps"),
])
def test_cache_copies_refuse(raw, kw, status, needle):
    _refused(raw, COPY, kw, status, needle)


@pytest.mark.parametrize("kw,needle", [(dict(v_codes=KC), "overlaps"), (dict(k_scales=KC + 4096), "overlaps"),
                                       (dict(starts=KC + 64), "starts")])
def test_append_refuses_aliased_caches(kw, needle):
    _refused(fastvr.kv4_append_raw, COPY, kw, INV, needle)


@pytest.mark.parametrize("kw", [dict(v=KN), dict(v=KN + 512), dict(k_st=512, k_sb=1536, v_st=512, v_sb=1536, v=KN + 256),
                                dict(k_st=512, k_sb=1536, v_st=512, v_sb=2048, v=KN + 512), dict(starts=KN + 64)])
def test_read_refuses_overlapping_outputs(kw):
    _refused(fastvr.kv4_read_raw, COPY, kw, INV, "overlaps")


@pytest.mark.parametrize("raw", [fastvr.kv4_append_raw, fastvr.kv4_read_raw], ids=["append", "read"])
@pytest.mark.parametrize("kw", [dict(B=0), dict(H=0), dict(n=0), dict(n=0, first=64), dict(n=0, k=None, v=None, k_codes=None)])
def test_cache_copies_empty(raw, kw):
    assert raw(*dict(COPY, **kw).values(), None) == fastvr.OK and fastvr.last_error() == ""


@pytest.mark.parametrize("kw,status,needle", [
    (dict(q=None), INV, "q is NULL"), (dict(o=None), INV, "o is NULL"), (dict(k_codes=None), INV, "k_codes is NULL"),
    (dict(v_scales=None), INV, "v_scales is NULL"), (dict(q=Q + 8), INV, "aligned"), (dict(o=O + 4), INV, "aligned"),
    (dict(lse=LSE + 2), INV, "lse"), (dict(lens=LENS + 1), INV, "lens"), (dict(workspace=WS + 8), INV, "workspace"),
    (dict(workspace=None), INV, "workspace"), (dict(workspace_bytes=64), INV, "workspace"), (dict(B=-1), INV, "negative"),
    (dict(cache_len=-1), INV, "negative"), (dict(d=80), UNS, "head_dim"), (dict(Hkv=3), INV, "multiple"), (dict(Hkv=0), INV, "multiple"),
    (dict(chunk_len=0), INV, "chunk_len"), (dict(window_chunks=-2), INV, "window_chunks"), (dict(capacity=8999), INV, "capacity"),
    (dict(capacity=1 << 25), UNS, "capacity"), (dict(cache_len=1 << 25, capacity=1 << 25), UNS, "cache_len"), (dict(scale=float("inf")), INV, "scale"),
    (dict(o_bf16=2), INV, "o_bf16"), (dict(q_st=500), INV, "token stride"), (dict(o_sb=512), INV, "batch stride"),
    (dict(Nq=1 << 31), UNS, "2^31"), (dict(H=65536, Hkv=65536), UNS, "65535"), (dict(H=32768, Hkv=32768, Nq=1 << 17), UNS, "2^31"), (dict(B=1 << 30), UNS, ""),
    (dict(o=Q), INV, "overlaps"), (dict(o=KC + 64), INV, "overlaps"), (dict(lse=O), INV, "overlaps"), (dict(workspace=VS), INV, "overlaps"),
    (dict(workspace=Q), INV, "overlaps"), (dict(lse=VC), INV, "overlaps"), (dict(lens=O + 8), INV, "overlaps"),
    (dict(q_st=1 << 31, q_sb=1 << 33), UNS, "strides"),
])
def test_attn_refuses(kw, status, needle):
    _refused(fastvr.kv4_attn_raw, ATTN, kw, status, needle)


@pytest.mark.parametrize("kw", [dict(B=0), dict(H=0, Hkv=0), dict(Nq=0), dict(Nq=0, q=None, o=None, k_codes=None, workspace=None)])
def test_attn_empty(kw):
    assert fastvr.kv4_attn_raw(*dict(ATTN, **kw).values(), None) == fastvr.OK and fastvr.last_error() == ""


def test_workspace_sizes():
    assert fastvr.kv4_attn_workspace(1, 12, 12, 1, 128, 100, 100) == 0
    need = fastvr.kv4_attn_workspace(1, 12, 12, 1, 128, 65280, 65280)
    assert need > 0 and need % (12 * (128 * 4 + 8)) == 0
    assert fastvr.kv4_attn_workspace(0, 12, 12, 1, 128, 65280, 65280) == 0
    for bad in [(1, 12, 5, 1, 128, 10, 10), (1, 12, 12, 1, 96, 10, 10), (1, 12, 12, 1, 128, 10, 0), (-1, 12, 12, 1, 128, 10, 10)]:
        with pytest.raises(fastvr.FastVRError):
            fastvr.kv4_attn_workspace(*bad)
    assert fastvr.load().fastvr_kv4_attn_workspace(1, 1, 1, 1, 128, 1, 1, -1, None) == INV
    n = ctypes.c_int64(7)
    assert fastvr.load().fastvr_kv4_attn_workspace(1, 1, 1, 1, 128, 1, 1, -3, ctypes.byref(n)) == INV and n.value == 7
