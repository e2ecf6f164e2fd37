"""Windowed attention and the quantised cache, without a GPU: what the entry points refuse (before anything is launched) and the sizes of
their buffers and workspaces."""
import ctypes

import pytest

from paper_2512_05754_amd import binding
from paper_2512_05754_amd.binding import UsvCache, UsvStrides, UsvWindow, UsvWindowGrads

FAKE = 0x7F0000001000  # aligned, not NULL; never followed, since the calls end before
AT_END = binding.USV_Q_AT_END
F32, BF16, F16 = binding.USV_F32, binding.USV_BF16, 2
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3


def window(**over):
    w = UsvWindow(2, 8, 4, 100, 300, 128, BF16, 50, 0, 1, 1, AT_END)
    for name, x in over.items():
        setattr(w, name, x)
    return w


def cache(**over):
    c = UsvCache(2, 4, 128, 4, 64, 40, 10, FAKE)
    for name, x in over.items():
        setattr(c, name, x)
    return c


def attn(w, q=FAKE, k=FAKE, v=FAKE, scale=0.0, out=FAKE, lse=FAKE, ws=None, ws_bytes=0):
    return binding.lib().usv_window_attn(q, k, v, None if w is None else ctypes.byref(w), scale, out, lse, ws, ws_bytes, None)


def backward(w, q=FAKE, k=FAKE, v=FAKE, out=FAKE, lse=FAKE, dout=FAKE, grads=UsvWindowGrads(), scale=0.0, dq=FAKE, dk=FAKE, dv=FAKE, ws=FAKE,
             ws_bytes=1 << 40):
    g = None if grads is None else ctypes.byref(grads)
    return binding.lib().usv_window_attn_backward(q, k, v, out, lse, dout, ctypes.byref(w), g, scale, dq, dk, dv, ws, ws_bytes, None)


def write(c, buffer=FAKE, k=FAKE, v=FAKE, dtype=BF16, rows=5, ks=None, vs=None, starts=FAKE, counts=None, read=False):
    f = binding.lib().usv_cache_read if read else binding.lib().usv_cache_write
    by = [None if s is None else ctypes.byref(s) for s in (ks, vs)]
    return f(buffer, None if c is None else ctypes.byref(c), k, v, dtype, rows, *by, starts, counts, None)


def attend(c, w, q=FAKE, buffer=FAKE, scale=0.0, out=FAKE, lse=FAKE, ws=None, ws_bytes=0):
    return binding.lib().usv_cache_attn(q, buffer, ctypes.byref(c), ctypes.byref(w), scale, out, lse, ws, ws_bytes, None)


def said():
    return binding.lib().usv_last_error().decode()


MOST = 1 << 30
BAD_WINDOWS = [
    (INVALID, dict(batch=0)), (INVALID, dict(q_heads=0)), (INVALID, dict(kv_heads=0)), (INVALID, dict(kv_heads=-4)), (INVALID, dict(kv_heads=3)),
    (INVALID, dict(q_heads=4, kv_heads=8)), (INVALID, dict(q_len=-1)), (INVALID, dict(kv_len=-1)), (INVALID, dict(q_len=MOST + 1)), (INVALID, dict(kv_len=MOST + 1)),
    (UNSUPPORTED, dict(head_dim=96)), (UNSUPPORTED, dict(head_dim=0)), (UNSUPPORTED, dict(dtype=F16)), (UNSUPPORTED, dict(dtype=-1)),
    (INVALID, dict(chunk=0)), (INVALID, dict(chunk=-5)), (INVALID, dict(chunk=MOST + 1)), (INVALID, dict(left=MOST + 1)), (INVALID, dict(right=MOST + 1)),
    (INVALID, dict(sinks=-1)), (INVALID, dict(sinks=MOST + 1)), (INVALID, dict(q_start=MOST + 1)), (INVALID, dict(q_start=-MOST - 1)), (INVALID, dict(seq_lens=FAKE + 2)),
    (UNSUPPORTED, dict(batch=8192)), (UNSUPPORTED, dict(batch=4096, q_len=1 << 24)),
]


@pytest.mark.parametrize("status,over", BAD_WINDOWS)
def test_bad_windows(status, over):
    w = window(**over)
    assert attn(w) == status and said()
    assert backward(w) == status
    assert binding.lib().usv_window_workspace_bytes(ctypes.byref(w)) == 0
    assert binding.lib().usv_window_backward_workspace_bytes(ctypes.byref(w)) == 0
    assert attend(cache(), w) != 0


def test_long_tables_are_no_reason_to_refuse():
    """Only the gradients have workgroups per key: many sequences with tables for a million positions are an ordinary decoding batch."""
    L = binding.lib()
    c = cache(batch=256, kv_heads=8, table_pages=16384)
    w = window(batch=256, q_heads=32, kv_heads=8, q_len=1, kv_len=1 << 20, left=-1, seq_lens=FAKE)
    assert L.usv_cache_attn_workspace_bytes(ctypes.byref(c), ctypes.byref(w)) >= 0
    assert attend(c, w, out=None) == INVALID and "out" in said()  # (as far as the pointers)
    assert attn(w, out=None) == INVALID and "out" in said()
    assert backward(window(batch=4096, kv_len=1 << 24)) == UNSUPPORTED and "kv_len" in said()
    assert L.usv_window_backward_workspace_bytes(ctypes.byref(window(batch=4096, kv_len=1 << 24))) == 0


def test_no_window():
    assert attn(None) == INVALID and "NULL" in said()
    assert binding.lib().usv_window_workspace_bytes(None) == 0
    assert binding.lib().usv_window_backward_workspace_bytes(None) == 0


BAD_STRIDES = [UsvStrides(-8, 12800, 128), UsvStrides(102400, 12800, 132), UsvStrides(102400, (1 << 40) + 8, 128), UsvStrides(102400, 12800, (1 << 28) + 8)]
OVERLAPS = [UsvStrides(0, 12800, 128), UsvStrides(102400, 0, 128), UsvStrides(102400, 12800, 64), UsvStrides(64, 12800, 128)]


@pytest.mark.parametrize("st", BAD_STRIDES)
@pytest.mark.parametrize("name", ["q", "k", "v", "out", "dout", "dq", "dk", "dv"])
def test_bad_strides(name, st):
    w, g = window(), UsvWindowGrads()
    setattr(w if hasattr(w, name) else g, name, st)
    if hasattr(w, name):
        assert attn(w) == INVALID and said().startswith(name + ":")
    assert backward(w, grads=g) == INVALID and said().startswith(name + ":")
    if name in ("k", "v"):
        for read in (False, True):
            assert write(cache(), **{name + "s": st}, read=read) == INVALID and said().startswith(name + ":")


@pytest.mark.parametrize("st", OVERLAPS)
def test_written_rows_do_not_overlap(st):
    assert attn(window(out=st)) == INVALID and "overlap" in said()
    assert attend(cache(), window(out=st, seq_lens=FAKE)) == INVALID and "overlap" in said()
    for name in ("dq", "dk", "dv"):
        assert backward(window(), grads=UsvWindowGrads(**{name: st})) == INVALID and "overlap" in said()
    for name in ("ks", "vs"):
        assert write(cache(), **{name: st}, read=True) == INVALID and "overlap" in said()


@pytest.mark.parametrize("bad", [None, FAKE + 8])
def test_pointers(bad):
    """NULL and not aligned to 16 bytes."""
    for name in ("q", "k", "v", "out"):
        assert attn(window(), **{name: bad}) == INVALID and name in said()
    for name in ("q", "k", "v", "out", "lse", "dout", "dq", "dk", "dv", "ws"):
        assert backward(window(), **{name: bad}) == INVALID and name in said()
    for read in (False, True):
        for name in ("k", "v", "starts"):
            assert write(cache(), **{name: bad}, read=read) == INVALID and name in said()
        assert write(cache(), buffer=bad, read=read) == INVALID and "cache" in said()
        assert write(cache(page_table=bad), read=read) == INVALID and "page_table" in said()
    w = window(seq_lens=FAKE)
    for name in ("q", "out"):
        assert attend(cache(), w, **{name: bad}) == INVALID and name in said()
    assert attend(cache(), w, buffer=bad) == INVALID and "cache" in said()
    assert attend(cache(page_table=bad), w) == INVALID and "page_table" in said()
    if bad:
        assert attn(window(), lse=bad) == INVALID and "lse" in said()
        assert attn(window(), ws=bad, ws_bytes=1 << 40) == INVALID and "ws" in said()
        assert attend(cache(), w, lse=bad) == INVALID and attend(cache(), w, ws=bad, ws_bytes=1 << 40) == INVALID
        assert write(cache(), counts=bad) == INVALID and write(cache(), counts=bad, read=True) == INVALID


def test_scales():
    for scale in (float("nan"), float("inf")):
        assert attn(window(), scale=scale) == INVALID and backward(window(), scale=scale) == INVALID
        assert attend(cache(), window(seq_lens=FAKE), scale=scale) == INVALID
        assert "scale" in said()


def test_workspaces():
    L = binding.lib()
    w = window(q_len=4, kv_len=50000, left=-1)  # few rows, long lists: shared out
    need = L.usv_window_workspace_bytes(ctypes.byref(w))
    assert need > 0 and need % 16 == 0
    assert attn(w, ws=FAKE, ws_bytes=need - 1) == WORKSPACE and str(need) in said()
    many = window(q_len=50000, kv_len=50000, left=-1)  # rows that fill the chip
    assert L.usv_window_workspace_bytes(ctypes.byref(many)) == 0
    for dtype in (BF16, F32):
        for x in (window(dtype=dtype), window(dtype=dtype, q_len=50000, kv_len=50000, left=-1), window(dtype=dtype, q_len=3, kv_len=9000, left=-1, right=-1)):
            n = L.usv_window_backward_workspace_bytes(ctypes.byref(x))
            assert n >= x.batch * x.q_heads * x.q_len * 4
            assert backward(x, ws_bytes=n - 1) == WORKSPACE and str(n) in said()
    assert L.usv_window_backward_workspace_bytes(ctypes.byref(window(q_len=0, kv_len=0))) > 0
    w = window(q_len=1, seq_lens=FAKE, kv_len=640, left=-1)
    assert L.usv_cache_attn_workspace_bytes(ctypes.byref(cache()), ctypes.byref(w)) == 0  # (a list too short to share out)
    c = cache(table_pages=1000)
    for rows in (1, 4000):  # pieces; a copy of the keys
        w = window(q_len=rows, seq_lens=FAKE, kv_len=64000, left=-1)
        need = L.usv_cache_attn_workspace_bytes(ctypes.byref(c), ctypes.byref(w))
        assert need > 0 and attend(c, w, ws=FAKE, ws_bytes=need - 1) == WORKSPACE and str(need) in said()


def test_workspace_does_not_grow_with_the_window():
    """Gradients keep a record per row and a bounded number of pieces: nothing of rows times keys."""
    for dtype in (BF16, F32):
        n = binding.lib().usv_window_backward_workspace_bytes(ctypes.byref(window(dtype=dtype, batch=1, q_len=100000, kv_len=100000, left=-1, right=-1)))
        assert n <= 8 * 100000 * 16 + 4096 * 2 * 128 * 128 * 4


BAD_CACHES = [
    (INVALID, dict(batch=0)), (INVALID, dict(kv_heads=0)), (UNSUPPORTED, dict(batch=16384)), (UNSUPPORTED, dict(head_dim=32)), (UNSUPPORTED, dict(bits=2)),
    (UNSUPPORTED, dict(bits=16)), (INVALID, dict(page_size=0)), (INVALID, dict(page_size=8)), (INVALID, dict(page_size=40)), (INVALID, dict(page_size=65552)),
    (INVALID, dict(pages=0)), (INVALID, dict(table_pages=0)), (INVALID, dict(table_pages=1 << 25)), (INVALID, dict(table_pages=-3)),
]


@pytest.mark.parametrize("status,over", BAD_CACHES)
def test_bad_caches(status, over):
    c = cache(**over)
    assert write(c) == status and said()
    assert write(c, read=True) == status
    assert binding.lib().usv_cache_bytes(ctypes.byref(c)) == 0
    assert attend(c, window(seq_lens=FAKE)) == status
    assert binding.lib().usv_cache_attn_workspace_bytes(ctypes.byref(c), ctypes.byref(window())) == 0


def test_cache_rows():
    assert write(None) == INVALID
    for read in (False, True):
        assert write(cache(), rows=-1, read=read) == INVALID
        assert write(cache(), rows=(1 << 26) + 1, read=read) == INVALID
        assert write(cache(), dtype=F16, read=read) == UNSUPPORTED
        assert write(cache(), rows=0, k=None, v=None, read=read) == 0  # (nothing to do is not an error)


@pytest.mark.parametrize("status,over", [
    (UNSUPPORTED, dict(dtype=F32)), (INVALID, dict(batch=3)), (INVALID, dict(kv_heads=8)), (INVALID, dict(head_dim=64)), (INVALID, dict(kv_len=641)),
    (INVALID, dict(q_start=0)), (INVALID, dict(seq_lens=None)), (INVALID, dict(seq_lens=FAKE + 1)),
])
def test_windows_that_do_not_fit_the_cache(status, over):
    w = window(seq_lens=FAKE)
    for name, x in over.items():
        setattr(w, name, x)
    assert attend(cache(), w) == status and said()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bits", [4, 8])
def test_cache_bytes(d, bits):
    """K codes, V codes, K scales, V scales of every page and head; beyond 4 GiB too."""
    per = 2 * (d * bits // 8 + d // 32)
    for pages, heads, page in ((1, 1, 16), (40, 4, 64), (100000, 8, 240)):
        assert binding.lib().usv_cache_bytes(ctypes.byref(cache(pages=pages, kv_heads=heads, head_dim=d, bits=bits, page_size=page))) == pages * heads * page * per


def test_nothing_to_do():
    assert attn(window(q_len=0), q=None, k=None, v=None, out=None, lse=None) == 0
    assert attend(cache(), window(q_len=0, seq_lens=FAKE), q=None, out=None, lse=None) == 0
