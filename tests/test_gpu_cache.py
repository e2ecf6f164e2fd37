"""The quantised cache on the GPU: what is written is read back exactly as the oracle has it, and attention over it.

Values read back are compared exactly: scales are powers of two, codes have at most four significant bits, so nothing rounds but the
quantisation itself.  cache_attn: bounds as in test_gpu_window.py (bf16), on the values that the cache holds.
"""
import numpy as np
import pytest
import torch

from oracle import window_oracle as wo
from test_gpu_window import close, close_lse, f64, normal

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def table(B, per, pages, seed=0):
    g = torch.Generator().manual_seed(seed)
    return torch.randperm(pages, generator=g)[: B * per].to(torch.int32).reshape(B, per)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bits", [4, 8])
def test_every_bf16_value_and_ties(usv, bits, dtype):
    """All finite bf16 values, each as its group's largest and beside larger ones; fp32: values at and next to the borders too."""
    x = torch.arange(0x7f80, dtype=torch.int32)
    x = torch.cat([x, x + 0x8000]).to(torch.int16).view(torch.bfloat16).float()
    rng = np.random.default_rng(1)
    rows = []
    for scale in (1.0, 0.5, 2.0 ** -20):
        g = np.outer(x.numpy(), rng.uniform(-1, 1, 32)).astype(np.float32) * np.float32(scale)
        g[:, 0] = x.numpy()
        rows.append(g)
    codes = wo.E2M1 if bits == 4 else wo.E4M3
    mid = (codes[1:] + codes[:-1]) / 2
    top = 7.0 if bits == 4 else 464.0
    edge = np.concatenate([codes, mid, mid * (1 + 2.0 ** -22), mid * (1 - 2.0 ** -22), [top, top * (1 + 2.0 ** -22), top * (1 - 2.0 ** -22)]])
    edge = np.concatenate([edge, -edge])
    edge = np.pad(edge, (0, -len(edge) % 31)).reshape(-1, 31)
    for s in (1.0, 2.0 ** 40, 2.0 ** -100, 3.0 / 2):
        rows.append(np.concatenate([np.full((len(edge), 1), codes[-1]), edge], 1) * s)
        rows.append(np.concatenate([np.zeros((len(edge), 1)), edge], 1) * s)
    flat = torch.from_numpy(np.concatenate(rows).astype(np.float32)).to(dtype)
    flat = flat[: len(flat) // 4 * 4].reshape(1, 1, -1, 128)
    n = flat.shape[2]
    per = -(-n // 64)
    cache = usv.cache_empty(per, 1, 64, 128, bits)
    t = table(1, per, per).to(DEV)
    v = flat.flip(2)
    usv.cache_write(cache, flat.to(DEV), v.to(DEV), t, ints([0]), bits=bits)
    k2, v2 = usv.cache_read(cache, t, ints([0]), n, head_dim=128, bits=bits, dtype=torch.float32)
    for got, src in ((k2, flat), (v2, v)):
        want = wo.cache_values(f64(src), bits)
        assert np.array_equal(f64(got), want), np.argwhere(f64(got) != want)[:3]
    k3, v3 = usv.cache_read(cache, t, ints([0]), n, head_dim=128, bits=bits)
    assert torch.equal(k3.float(), k2) and torch.equal(v3.float(), v2)


@pytest.mark.parametrize("page", [16, 48, 64, 240])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bits", [4, 8])
def test_places_layout_and_strides(usv, bits, d, page):
    """Rows land where the layout says, from strided views of a projection, starts inside a page; the rest of the buffer is left as it was."""
    B, H, n, L = 2, 3, 77, 300
    per = -(-L // page)
    pages = B * per + 3
    t = table(B, per, pages, seed=page)
    x = normal((B, n, 2, H, d), 3, torch.bfloat16)
    k, v = (x[:, :, i].transpose(1, 2) for i in range(2))
    cache = usv.cache_empty(pages, H, page, d, bits).fill_(0xA5)
    before = cache.cpu().numpy().copy()
    starts, counts = [L - n, 5], [n, 40]
    usv.cache_write(cache, k.to(DEV), v.to(DEV), t.to(DEV), ints(starts), bits=bits, counts=ints(counts))
    buf = cache.cpu().numpy()
    untouched = np.ones(buf.shape, dtype=bool)
    cb, sb = d * bits // 8, d // 32
    for b in range(B):
        for i in range(counts[b]):
            pos = starts[b] + i
            pg, row = int(t[b, pos // page]), pos % page
            for which, src in enumerate((k, v)):
                untouched[pg, :, (which * page + row) * cb:][:, :cb] = False
                untouched[pg, :, 2 * page * cb + (which * page + row) * sb:][:, :sb] = False
                for h in range(H):
                    got = wo.cache_decode(buf, pg, row, h, which, page, d, bits)
                    assert np.array_equal(got, wo.cache_values(f64(src[b, h, i]), bits)), (b, i, h, which)
    assert np.array_equal(buf[untouched], before[untouched])
    # read: into views, rows beyond counts left as they were
    big = torch.full((B, n, 2, H, d + 8), 9.0, dtype=torch.bfloat16, device=DEV)
    ko, vo = (big[:, :, i, :, :d].transpose(1, 2) for i in range(2))
    usv.cache_read(cache, t.to(DEV), ints(starts), n, head_dim=d, bits=bits, counts=ints(counts), k=ko, v=vo)
    for src, got in ((k, ko), (v, vo)):
        for b in range(B):
            assert np.array_equal(f64(got[b, :, : counts[b]]), wo.cache_values(f64(src[b, :, : counts[b]]), bits))
            assert bool((got[b, :, counts[b]:] == 9).all())
    assert bool((big[..., d:] == 9).all())


@pytest.mark.parametrize("bits", [4, 8])
def test_all_codes_under_all_scales(usv, bits):
    """A buffer of every code under every scale byte the format has."""
    codes = np.arange(256, dtype=np.uint8)
    if bits == 8:
        codes = codes[(codes & 0x7f) != 0x7f]  # (NaN codes are never written)
    lo, hi = (2, 252) if bits == 4 else (10, 246)  # e = -125 .. 125, -117 .. 119: the least and largest code stay normal numbers
    cb = 128 * bits // 8
    rows = []
    line = np.resize(codes, -(-len(codes) // cb) * cb).reshape(-1, cb)
    scales = np.arange(lo, hi + 1, dtype=np.uint8)
    scales = np.resize(scales, (-(-len(scales) // 4), 4))
    for s in scales:
        rows += [(c, s) for c in line]
    n, page = len(rows), 16
    per = -(-n // page)
    buf = np.zeros((per, 1, 2 * page * (cb + 4)), dtype=np.uint8)
    for i, (c, s) in enumerate(rows):
        pg, row = divmod(i, page)
        for which in range(2):
            buf[pg, 0, (which * page + row) * cb:][:cb] = c
            buf[pg, 0, 2 * page * cb + (which * page + row) * 4:][:4] = s
    t = torch.arange(per, dtype=torch.int32)[None].to(DEV)
    got = usv.cache_read(torch.from_numpy(buf).to(DEV), t, ints([0]), n, head_dim=128, bits=bits, dtype=torch.float32)
    for which in range(2):
        want = np.stack([wo.cache_decode(buf, i // page, i % page, 0, which, page, 128, bits) for i in range(n)])
        assert np.array_equal(f64(got[which][0, 0]), want)


@pytest.mark.parametrize("bits", [4, 8])
def test_not_finite_groups_and_zeros(usv, bits):
    x = normal((1, 1, 6, 64), 5, torch.float32)
    x[0, 0, 0, 3] = float("inf")
    x[0, 0, 1, 40] = float("nan")
    x[0, 0, 2] = 0
    x[0, 0, 3, :32] = 1e-40
    x[0, 0, 4] = torch.tensor(3.3e38)
    cache = usv.cache_empty(1, 1, 16, 64, bits)
    t = ints([[0]])
    for dtype in (torch.float32, torch.bfloat16):
        y = x.to(dtype)
        usv.cache_write(cache, y.to(DEV), y.to(DEV), t, ints([0]), bits=bits)
        k, v = usv.cache_read(cache, t, ints([0]), 6, head_dim=64, bits=bits, dtype=dtype)
        want = wo.cache_values(f64(y), bits)
        assert np.isnan(want[0, 0, 0, :32]).all() and np.isfinite(want[0, 0, 0, 32:]).all()
        for got in (k, v):
            assert np.array_equal(f64(got), want, equal_nan=True)


def test_bad_places(usv):
    """Positions outside the table and page ids outside the buffer: not written, read as zeros."""
    d, page = 64, 16
    k = normal((3, 2, 40, d), 6, torch.bfloat16).to(DEV)
    cache = usv.cache_empty(4, 2, page, d).fill_(0)
    t = ints([[0, -1, 1], [2, 99, 3], [1 << 30, -(1 << 31), 4]])
    usv.cache_write(cache, k, k, t, ints([-7, 20, 0]))
    got, _ = usv.cache_read(cache, t, ints([-7, 20, 0]), 40, head_dim=d)
    want = wo.cache_values(f64(k), 4)
    pos = np.arange(40)[None] + np.array([-7, 20, 0])[:, None]
    for b in range(3):
        for i in range(40):
            slot = pos[b, i] // page if 0 <= pos[b, i] < 3 * page else None
            ok = slot is not None and 0 <= int(t[b, slot]) < 4
            assert np.array_equal(f64(got[b, :, i]), want[b, :, i] if ok else np.zeros((2, d))), (b, i)


class Decode:
    def __init__(self, B, Hq, Hkv, Lq, cap, d, bits, page, lens, left=-1, right=0, sinks=0, chunk=1):
        self.B, self.Hq, self.Hkv, self.Lq, self.cap, self.d, self.bits, self.page, self.lens = B, Hq, Hkv, Lq, cap, d, bits, page, lens
        self.args = dict(left=left, right=right, sinks=sinks, chunk=chunk)
        self.M = wo.masks(B, Lq, cap, left, right, sinks, chunk, None, lens)

    def __repr__(self):
        return "-".join(str(x) for x in (self.B, self.Hq, self.Hkv, self.Lq, self.cap, self.d, self.bits, self.page, self.lens, *self.args.values())).replace(" ", "")


DECODES = [
    Decode(1, 1, 1, 1, 16, 128, 4, 16, [1]),
    Decode(2, 2, 2, 1, 48, 64, 8, 48, [48, 0]),
    Decode(3, 8, 2, 1, 320, 128, 4, 64, [301, 17, 64]),
    Decode(2, 8, 1, 1, 4096, 64, 4, 64, [4095, 1500]),                    # keys shared out
    Decode(1, 4, 4, 1, 2048, 128, 8, 128, [2048], 700, 0, 4),             # window and sinks, shared out
    Decode(2, 4, 2, 5, 240, 128, 4, 240, [230, 3], 60, 0, 2),             # five new tokens, a sequence shorter than they are
    Decode(1, 16, 2, 3, 400, 64, 8, 16, [399], 33, 0, 40),                # sinks that end inside a page, 24 rows a key head
    Decode(1, 2, 2, 90, 320, 128, 4, 64, [305], 1, 0, 1, 45),             # two frames of 45 tokens against window and first frame
    Decode(1, 3, 1, 50, 224, 64, 4, 32, [200], -1, -1),                   # both ways, 150 rows
    Decode(2, 2, 1, 70, 256, 128, 8, 64, [256, 71], 0, 1, 0, 16),
    Decode(1, 1, 1, 1, 640, 64, 4, 64, [600], 0, 0, 0),                   # sees itself only
    # 1024 rows a key head and more: the keys that they see are taken out first
    Decode(2, 4, 1, 300, 960, 128, 4, 64, [960, 310], 1, 0, 1, 150),
    Decode(1, 1, 1, 1100, 2560, 64, 8, 16, [2500], 100, 0, 3),
    Decode(1, 2, 1, 520, 640, 128, 8, 64, [600]),
    Decode(2, 8, 2, 256, 2048, 64, 4, 256, [2000, 0], 1, 0, 2, 128),
]


@pytest.mark.parametrize("c", DECODES, ids=repr)
def test_attention_over_the_cache(usv, c):
    """Against the oracle on the values the cache holds.  What no query sees is NaN, and pages that hold only such rows have no valid id."""
    per = c.cap // c.page
    pages = c.B * per
    k, v = (normal((c.B, c.Hkv, c.cap, c.d), 10 + i, torch.bfloat16) * 1.5 for i in range(2))
    q = normal((c.B, c.Hq, c.Lq, c.d), 12, torch.bfloat16)
    seen, live = c.M.any(1), c.M.any(2)
    q = torch.where(torch.from_numpy(live)[:, None, :, None], q, torch.tensor(float("nan"), dtype=q.dtype))
    kq, vq = (wo.cache_values(f64(x), c.bits) for x in (k, v))
    nan = torch.tensor(float("nan"), dtype=k.dtype)
    s4 = torch.from_numpy(seen)[:, None, :, None]
    cache = usv.cache_empty(pages, c.Hkv, c.page, c.d, c.bits).fill_(0xFF)
    t = table(c.B, per, pages, seed=3)
    usv.cache_write(cache, torch.where(s4, k, nan).to(DEV), torch.where(s4, v, nan).to(DEV), t.to(DEV), torch.zeros(c.B, dtype=torch.int32, device=DEV), bits=c.bits)
    used = torch.from_numpy(seen).reshape(c.B, per, c.page).any(2)
    t = torch.where(used, t, torch.tensor(1 << 30, dtype=torch.int32))
    ref, lse_ref, mag = wo.window_attn(f64(q), kq, vq, c.M)
    out, lse = usv.cache_attn(q.to(DEV), cache, t.to(DEV), ints(c.lens), **c.args, bits=c.bits, return_lse=True)
    close(out, ref, mag, "bf16", "out")
    close_lse(lse, lse_ref)
    if c.Lq * (c.Hq // c.Hkv) >= 1024:  # without scratch the codes are read where they lie
        out2, lse2 = usv.cache_attn(q.to(DEV), cache, t.to(DEV), ints(c.lens), **c.args, bits=c.bits, return_lse=True, workspace=torch.empty(0, dtype=torch.uint8, device=DEV))
        close(out2, ref, mag, "bf16", "out")
        close_lse(lse2, lse_ref)
    # queries as a projection lays them out, the output into such a view: the same bits
    buf = torch.full((c.B, c.Lq, c.Hq, c.d + 8), 7.0, dtype=q.dtype, device=DEV)
    qs = q.transpose(1, 2).contiguous().transpose(1, 2).to(DEV)
    usv.cache_attn(qs, cache, t.to(DEV), ints(c.lens), **c.args, bits=c.bits, out=buf[..., : c.d].transpose(1, 2))
    assert torch.equal(buf[..., : c.d].transpose(1, 2), out) and bool((buf[..., c.d:] == 7).all())


def test_a_cache_beyond_32_bit_offsets(usv):
    """A buffer of more than 4 GiB, the rows in its last pages."""
    d, page, H, bits = 128, 64, 8, 8
    pages = (9 << 29) // (H * 2 * page * (d + 4)) + 1
    cache = usv.cache_empty(pages, H, page, d, bits)
    assert cache.numel() > 1 << 32
    n = 200
    t = torch.tensor([[pages - 1, pages - 3, 0, pages - 2]], dtype=torch.int32)
    k, v = (normal((1, H, n, d), 20 + i, torch.bfloat16) for i in range(2))
    usv.cache_write(cache, k.to(DEV), v.to(DEV), t.to(DEV), ints([0]), bits=bits)
    kr, vr = usv.cache_read(cache, t.to(DEV), ints([0]), n, head_dim=d, bits=bits)
    kq, vq = (wo.cache_values(f64(x), bits) for x in (k, v))
    assert np.array_equal(f64(kr), kq) and np.array_equal(f64(vr), vq)
    q = normal((1, H, 1, d), 22, torch.bfloat16)
    ref, _, mag = wo.window_attn(f64(q), kq, vq, wo.masks(1, 1, n, -1, 0, 0, 1))
    close(usv.cache_attn(q.to(DEV), cache, t.to(DEV), ints([n]), bits=bits), ref, mag, "bf16", "out")


def test_many_sequences_with_long_tables(usv):
    """Tables for a million positions each, of which a few are used: as with tables that just fit."""
    B, Hq, Hkv, d, page, n = 96, 16, 2, 64, 64, 150
    per = -(-n // page)
    cache = usv.cache_empty(B * per, Hkv, page, d, 4)
    short = table(B, per, B * per, seed=30).to(DEV)
    long = torch.zeros((B, (1 << 20) // page), dtype=torch.int32, device=DEV)
    long[:, :per] = short
    k, v = (normal((B, Hkv, n, d), 31 + i, torch.bfloat16) for i in range(2))
    q = normal((B, Hq, 1, d), 33, torch.bfloat16)
    usv.cache_write(cache, k.to(DEV), v.to(DEV), long, ints([0] * B))
    lens = ints([n - b for b in range(B)])
    kq, vq = (wo.cache_values(f64(x), 4) for x in (k, v))
    M = wo.masks(B, 1, n, -1, 0, 0, 1, lens=[n - b for b in range(B)])
    ref, lse_ref, mag = wo.window_attn(f64(q), kq, vq, M)
    for t in (short, long):
        out, lse = usv.cache_attn(q.to(DEV), cache, t, lens, return_lse=True)
        close(out, ref, mag, "bf16", "out")
        close_lse(lse, lse_ref)


@pytest.mark.parametrize("bits", [4, 8])
def test_generation_frame_after_frame(usv, bits):
    """The operators as a streaming step uses them, captured once and replayed: write the new frame, attend to window and first frame over
    the cache.  Each step equals window_attn on what cache_read takes out, within the rounding of the weights, and the oracle."""
    B, H, T, d, page, frames = 2, 4, 24, 128, 16, 6
    args = dict(left=2, right=0, sinks=1, chunk=T)
    cap = frames * T
    t = table(B, cap // page, B * cap // page, seed=9).to(DEV)
    cache = usv.cache_empty(B * cap // page, H, page, d, bits)
    q, k, v = (torch.zeros((B, H, T, d), dtype=torch.bfloat16, device=DEV) for _ in range(3))
    starts, lens = ints([0] * B), ints([T] * B)
    out = torch.empty_like(q)
    ws = torch.empty(max(16, usv.cache_attn_workspace_bytes(q, cache, t, **args, bits=bits)), dtype=torch.uint8, device=DEV)

    def step():
        usv.cache_write(cache, k, v, t, starts, bits=bits)
        usv.cache_attn(q, cache, t, lens, **args, bits=bits, out=out, workspace=ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    all_k, all_v = [], []
    for f in range(frames):
        new = [normal((B, H, T, d), 100 * f + i, torch.bfloat16) for i in range(3)]
        for dst, src in zip((q, k, v), new):
            dst.copy_(src)
        all_k.append(wo.cache_values(f64(new[1]), bits))
        all_v.append(wo.cache_values(f64(new[2]), bits))
        starts.fill_(f * T)
        lens.fill_((f + 1) * T)
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        K, V = np.concatenate(all_k, 2), np.concatenate(all_v, 2)
        ref, _, mag = wo.window_attn(f64(new[0]), K, V, wo.masks(B, T, K.shape[2], **args))
        close(out, ref, mag, "bf16", f"frame {f}")
        kr, vr = usv.cache_read(cache, t, ints([0] * B), (f + 1) * T, head_dim=d, bits=bits)
        assert np.array_equal(f64(kr), K) and np.array_equal(f64(vr), V)
        close(usv.window_attn(q, kr, vr, **args), ref, mag, "bf16", f"frame {f}, read back")


def test_refusals(usv):
    q = torch.zeros((2, 4, 1, 64), dtype=torch.bfloat16, device=DEV)
    cache = usv.cache_empty(4, 2, 16, 64)
    t, lens = ints([[0, 1], [2, 3]]), ints([20, 3])
    k = torch.zeros((2, 2, 3, 64), dtype=torch.bfloat16, device=DEV)
    usv.cache_attn(q, cache, t, lens)
    for bad in (lambda: usv.cache_empty(4, 2, 15, 64), lambda: usv.cache_empty(4, 2, 16, 96), lambda: usv.cache_empty(4, 2, 16, 64, bits=5),
                lambda: usv.cache_empty(0, 2, 16, 64), lambda: usv.cache_attn(q, cache[:, :, 1:], t, lens), lambda: usv.cache_attn(q, cache, t, lens[:1]),
                lambda: usv.cache_write(cache, k[:, :1], k[:, :1], t, lens), lambda: usv.cache_write(cache, k, k[:, :, :2], t, lens),
                lambda: usv.cache_read(cache, t, lens, 3, head_dim=64, k=k[:, :, :2]), lambda: usv.cache_attn(q, cache, t[0], lens),
                lambda: usv.cache_attn(q, cache, t, lens, bits=16)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: usv.cache_attn(q.cpu(), cache, t, lens), lambda: usv.cache_attn(q, cache.cpu(), t, lens), lambda: usv.cache_attn(q, cache, t.long(), lens),
                lambda: usv.cache_write(cache, k.half(), k.half(), t, lens), lambda: usv.cache_write(cache.view(torch.int8), k, k, t, lens)):
        with pytest.raises(TypeError):
            bad()
    for status, bad in ((2, lambda: usv.cache_attn(q.float(), cache, t, lens)), (1, lambda: usv.cache_attn(q[:, :3], cache, t, lens)),
                        (1, lambda: usv.cache_attn(q, cache, t, lens, chunk=0))):
        with pytest.raises(usv.UsvError) as e:
            bad()
        assert e.value.status == status
    q1 = torch.zeros((1, 4, 1, 64), dtype=torch.bfloat16, device=DEV)
    big, tb = usv.cache_empty(64, 2, 64, 64), torch.arange(64, dtype=torch.int32, device=DEV)[None]
    assert usv.cache_attn_workspace_bytes(q1, big, tb) > 0
    with pytest.raises(usv.UsvError) as e:
        usv.cache_attn(q1, big, tb, ints([4000]), workspace=torch.empty(64, dtype=torch.uint8, device=DEV))
    assert e.value.status == 3
