"""Windowed attention with sinks and its gradient on the GPU, against the oracle in 64 bits.

Bounds.  bf16: a weight P (gradient: P or dS) is rounded to bf16 once, by at most half a step, 2^-8 of itself, and the result once more:
|error| <= 2^-8 (sum of |P| |v| + |result|), plus 1e-5 of that sum for the fp32 arithmetic around it (sums of up to 128 products of
24-bit accuracy in the logits, exp2 of their difference).  fp32: 1e-5 of the sum alone.  lse: fp32 on both, 1e-5 (1 + |lse|).
In the gradient dout.v and D are fp32 sums of up to 128 products that may cancel (a row that sees one key has dout.v = D): each is off by
up to 128 * 2^-24 = 7.6e-6 of its sum of absolute products, whatever is left, so 1e-5 of what those sums weigh is added for both types.
bf16 takes D from the rounded out first, off by 2^-8 of its products at most, and takes what is too much off again in proportion to rounded
weights, whose sum is 1 to 2^-8: what is left of it is at most three times 2^-16 of the products, for which 2^-14 is added.
"""
import numpy as np
import pytest
import torch

from oracle import window_oracle as wo

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = 2.0 ** -8


class Case:
    def __init__(self, B, Hq, Hkv, Lq, Lk, d, left, right=0, sinks=0, chunk=1, start=None, lens=None):
        self.B, self.Hq, self.Hkv, self.Lq, self.Lk, self.d = B, Hq, Hkv, Lq, Lk, d
        self.args = dict(left=left, right=right, sinks=sinks, chunk=chunk)
        self.start, self.lens = start, lens
        self.M = wo.masks(B, Lq, Lk, left, right, sinks, chunk, start, lens)

    def __repr__(self):
        return "-".join(str(x) for x in (self.B, self.Hq, self.Hkv, self.Lq, self.Lk, self.d, *self.args.values(), self.start, self.lens)).replace(" ", "")


CASES = [
    Case(1, 1, 1, 1, 1, 128, -1),                                    # one token
    Case(1, 2, 1, 1, 70, 64, 5, 0, 2),                               # one query over a cache
    Case(1, 2, 2, 64, 64, 128, -1),                                  # plain causal
    Case(2, 2, 2, 65, 65, 64, -1, -1),                               # everything, one past a tile
    Case(1, 4, 2, 130, 130, 128, 20, 0, 4),                          # window and sinks
    Case(1, 3, 1, 200, 333, 64, 31, 3, 40),                          # newest queries, three heads on one key head
    Case(2, 4, 4, 127, 127, 128, 1, 0, 1, 20),                       # frames
    Case(1, 2, 2, 190, 190, 64, 1, 1, 1, 33),                        # frames both ways, a cut last one
    Case(3, 2, 1, 100, 100, 128, 9, 0, 3, 1, 0, [100, 1, 0]),        # padded batch, one empty sequence
    Case(3, 2, 2, 40, 150, 64, -1, 0, 0, 1, None, [150, 64, 17]),    # padded batch, newest queries; rows before the first token
    Case(1, 1, 1, 50, 30, 128, -1, 0, 0, 1, -10, None),              # rows before and behind the sequence
    Case(1, 1, 1, 20, 300, 64, 0, 0, 200, 1, 250, None),             # sinks that reach far, a window of one
    Case(1, 2, 2, 257, 257, 128, 300, 300, 5, 7),                    # limits beyond the sequence
    Case(1, 1, 1, 70, 70, 64, 1 << 30, 1 << 30, 1 << 30, 1 << 30),   # the largest numbers
    Case(1, 8, 2, 3, 700, 128, -1, 0, 0),                            # few rows: the keys are shared out
    Case(2, 8, 1, 1, 1300, 64, 1000, 0, 8, 1, None, [1300, 600]),
]


def normal(shape, seed, dtype):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g, dtype=torch.float32).to(dtype)


def inputs(c, dtype, seed=0, gain=1.5):
    q = (normal((c.B, c.Hq, c.Lq, c.d), seed, torch.float32) * gain).to(dtype)
    k, v, = (normal((c.B, c.Hkv, c.Lk, c.d), seed + s, dtype) for s in (1, 2))
    do = normal((c.B, c.Hq, c.Lq, c.d), seed + 3, dtype)
    # what nobody sees may hold anything
    seen, live = torch.from_numpy(c.M.any(1))[:, None, :, None], torch.from_numpy(c.M.any(2))[:, None, :, None]
    bad = torch.tensor(float("nan"), dtype=dtype)
    return torch.where(live, q, bad), torch.where(seen, k, -bad), torch.where(seen, v, torch.tensor(float("inf"), dtype=dtype)), torch.where(live, do, bad)


def f64(t):
    return t.double().cpu().numpy()


def lens_of(c):
    return None if c.lens is None else torch.tensor(c.lens, dtype=torch.int32, device=DEV)


def close(got, ref, mag, dtype, what, terms=0.0):
    got = f64(got)
    assert np.isfinite(got).all(), what
    bound = 1e-5 * mag + (1e-5 + (2.0 ** -14 if dtype == "bf16" else 0.0)) * terms + (HALF_STEP * (mag + np.abs(ref)) if dtype == "bf16" else 0.0) + 1e-30
    off = np.abs(got - ref) / bound
    assert off.max(initial=0.0) <= 1.0, f"{what}: {off.max():.3g} of the bound at {np.unravel_index(off.argmax(), off.shape)}"


def close_lse(got, ref, what="lse"):
    got = f64(got)
    assert np.array_equal(np.isinf(got), np.isinf(ref)) and not np.isnan(got).any(), what
    fine = np.isfinite(ref)
    off = np.abs(got[fine] - ref[fine])
    assert (off <= 1e-5 * (1 + np.abs(ref[fine]))).all(), (what, off.max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", CASES, ids=repr)
def test_forward(usv, c, dtype):
    q, k, v, _ = inputs(c, TYPES[dtype])
    ref, lse_ref, mag = wo.window_attn(f64(q), f64(k), f64(v), c.M)
    out, lse = usv.window_attn(q.to(DEV), k.to(DEV), v.to(DEV), **c.args, q_start=c.start, seq_lens=lens_of(c), return_lse=True)
    close(out, ref, mag, dtype, "out")
    close_lse(lse, lse_ref)
    assert (f64(out)[~np.broadcast_to(c.M.any(2)[:, None], out.shape[:3])] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", CASES, ids=repr)
def test_backward(usv, c, dtype):
    q, k, v, do = inputs(c, TYPES[dtype], seed=10)
    ref, lse_ref, _ = wo.window_attn(f64(q), f64(k), f64(v), c.M)
    # `out` as the forward pass leaves it: rounded to the type
    out = torch.from_numpy(ref).to(TYPES[dtype])
    lse = torch.from_numpy(lse_ref).float()
    want, mags, terms = wo.window_attn_backward(f64(q), f64(k), f64(v), f64(do), c.M)
    got = usv.window_attn_backward(*(t.to(DEV) for t in (q, k, v, out, lse, do)), **c.args, q_start=c.start, seq_lens=lens_of(c))
    for name, x, r, m, e in zip(("dq", "dk", "dv"), got, want, mags, terms):
        close(x, r, m, dtype, name, e)
    assert (f64(got[0])[~np.broadcast_to(c.M.any(2)[:, None], q.shape[:3])] == 0).all()
    for x in got[1:]:
        assert (f64(x)[~np.broadcast_to(c.M.any(1)[:, None], k.shape[:3])] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradient_against_differences(usv, dtype):
    """The gradient of sum(out * weight) along a direction, against the difference of 64-bit forward passes."""
    c = Case(1, 4, 2, 90, 90, 64, 25, 0, 3)
    q, k, v, w = inputs(c, TYPES[dtype], seed=20)
    out, lse = usv.window_attn(q.to(DEV), k.to(DEV), v.to(DEV), **c.args, return_lse=True)
    got = usv.window_attn_backward(q.to(DEV), k.to(DEV), v.to(DEV), out, lse, w.to(DEV), **c.args)
    X = [f64(t) for t in (q, k, v)]
    rng, eps = np.random.default_rng(5), 1e-5
    for i in range(3):
        u = rng.standard_normal(X[i].shape)
        f = [(wo.window_attn(*[x + (s * eps * u if j == i else 0) for j, x in enumerate(X)], c.M)[0] * f64(w)).sum() for s in (1, -1)]
        slope = (f[0] - f[1]) / (2 * eps)
        g = f64(got[i])
        # each entry is off by its own rounding errors, which a direction of independent signs adds up in squares: of entries off by
        # 4 half steps (P or dS, out in D, the result; one more for slack) six deviations are never met
        tol = 6 * np.sqrt(((4 * (HALF_STEP if dtype == "bf16" else 1e-5) * np.abs(g).max()) ** 2 * u ** 2).sum()) + 1e-6 * abs(slope)
        assert abs((g * u).sum() - slope) <= tol, (i, (g * u).sum(), slope, tol)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_strides(usv, d, dtype):
    """Views of projections, of a packed qkv, expanded heads, and outputs that are views: the same bits as contiguous tensors."""
    B, H, L = 2, 4, 150
    a = dict(left=40, right=0, sinks=6)
    x = normal((B, L, 3, H, d), 30, TYPES[dtype]).to(DEV)
    q, k, v = (x[:, :, i].transpose(1, 2) for i in range(3))
    k1 = k[:, :1].expand(B, H, L, d)
    want = usv.window_attn(q.contiguous(), k1.contiguous(), v.contiguous(), **a, return_lse=True)
    buf = torch.full((B, L, H, d + 16), 7.0, dtype=TYPES[dtype], device=DEV)
    out = buf[..., :d].transpose(1, 2)
    got = usv.window_attn(q, k1, v, **a, out=out, return_lse=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert bool((buf[..., d:] == 7).all())
    do = normal((B, L, H, d), 31, TYPES[dtype]).to(DEV).transpose(1, 2)
    g = usv.window_attn_backward(q.contiguous(), k1.contiguous(), v.contiguous(), *want, do.contiguous(), **a)
    bufs = [torch.full((B, L, H, d + 16), 7.0, dtype=TYPES[dtype], device=DEV) for _ in range(3)]
    views = [b[..., :d].transpose(1, 2) for b in bufs]
    g2 = usv.window_attn_backward(q, k1, v, out, want[1], do, **a, dq=views[0], dk=views[1], dv=views[2])
    for x, y, b in zip(g, g2, bufs):
        assert torch.equal(x, y) and bool((b[..., d:] == 7).all())


def torch_rows(q, k, v, M, scale):
    """out, lse and sum P |v| of one head in 64 bits on the GPU: q [Lq, d], k, v [Lk, d], M [Lq, Lk]."""
    x = (q.double() @ k.double().T * scale).masked_fill(~M, -float("inf"))
    lse = torch.logsumexp(x, 1)
    P = torch.exp(x - lse[:, None])
    return P @ v.double(), lse, P @ v.double().abs()


@pytest.mark.parametrize("d, left, right, sinks, chunk", [(128, 2200, 0, 70, 1), (128, 3, 2, 1, 517), (64, 4200, 0, 3, 1), (64, 5, 1, 0, 700)])
def test_long_windows_of_many_rows(usv, d, left, right, sinks, chunk):
    """Launches of more than a round of workgroups with windows of more than a MiB: the keys are walked in a circle."""
    H, L = 17, 6400
    q, k, v = (normal((1, H, L, d), 200 + i, torch.bfloat16).to(DEV) for i in range(3))
    out, lse = usv.window_attn(q, k, v, left, right, sinks, chunk, return_lse=True)
    M = torch.from_numpy(wo.masks(1, L, L, left, right, sinks, chunk)[0]).to(DEV)
    for h in (0, 3, 7, 16):
        ref, ls, mag = torch_rows(q[0, h], k[0, h], v[0, h], M, d ** -0.5)
        close(out[0, h], f64(ref), f64(mag), "bf16", f"head {h}")
        close_lse(lse[0, h], f64(ls))
    again = usv.window_attn(q, k, v, left, right, sinks, chunk, return_lse=True)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H, L", [(3, 1100), (24, 1500)])
@pytest.mark.parametrize("left, right, sinks, chunk", [(-1, 0, 0, 1), (-1, -1, 0, 1), (300, 0, 100, 1), (1, 1, 1, 130), (40, 3, 64, 1)])
def test_workgroups_of_four_waves_and_of_two(usv, d, H, L, left, right, sinks, chunk):
    """54 and 576 workgroups: fewer and more than there are places; lists of two to twenty-four tiles, not shared out."""
    q, k, v = (normal((1, H, L, d), 230 + i, torch.bfloat16).to(DEV) for i in range(3))
    none = torch.empty(0, dtype=torch.uint8, device=DEV)
    out, lse = usv.window_attn(q, k, v, left, right, sinks, chunk, workspace=none, return_lse=True)
    M = torch.from_numpy(wo.masks(1, L, L, left, right, sinks, chunk)[0]).to(DEV)
    for h in range(0, H, 2):
        ref, ls, mag = torch_rows(q[0, h], k[0, h], v[0, h], M, d ** -0.5)
        close(out[0, h], f64(ref), f64(mag), "bf16", f"head {h}")
        close_lse(lse[0, h], f64(ls))


@pytest.mark.parametrize("d", [64, 128])
def test_long_windows_of_few_rows(usv, d):
    """In one piece and shared out, from one row to a block and a bit, the first key of the list at any place of a tile."""
    L, left = 5000, 4300
    k, v = (normal((1, 1, L, d), 210 + i, torch.bfloat16).to(DEV) for i in range(2))
    for n in (1, 63, 65, 130):
        q = normal((1, 2, n, d), 220 + n, torch.bfloat16).to(DEV)
        for sinks in (0, 1, 64, 200):
            M = torch.from_numpy(wo.masks(1, n, L, left, 0, sinks, 1)[0]).to(DEV)
            for ws in (None, torch.empty(0, dtype=torch.uint8, device=DEV)):
                out, lse = usv.window_attn(q, k, v, left, 0, sinks, workspace=ws, return_lse=True)
                for h in range(2):
                    ref, ls, mag = torch_rows(q[0, h], k[0, 0], v[0, 0], M, d ** -0.5)
                    close(out[0, h], f64(ref), f64(mag), "bf16", f"{n} rows, {sinks} sinks")
                    close_lse(lse[0, h], f64(ls))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq, Hkv, Lq, Lk, left, right, sinks, chunk", [
    (2, 1, 1500, 1500, 300, 0, 40, 1),    # lists of rows shared out, those of the sinks in more pieces
    (1, 1, 70, 5000, 4300, 0, 10, 1),     # lists of keys shared out
    (3, 1, 900, 2300, 2, 1, 1, 250),
    (8, 2, 40, 3000, -1, 0, 0, 1),
])
def test_gradients_of_long_lists(usv, d, dtype, Hq, Hkv, Lq, Lk, left, right, sinks, chunk):
    a = dict(left=left, right=right, sinks=sinks, chunk=chunk)
    q, do = (normal((1, Hq, Lq, d), 300 + i, TYPES[dtype]).to(DEV) for i in range(2))
    k, v = (normal((1, Hkv, Lk, d), 310 + i, TYPES[dtype]).to(DEV) for i in range(2))
    out, lse = usv.window_attn(q, k, v, **a, return_lse=True)
    dq, dk, dv = usv.window_attn_backward(q, k, v, out, lse, do, **a)
    M = torch.from_numpy(wo.masks(1, Lq, Lk, left, right, sinks, chunk)[0]).to(DEV)
    scale, G = d ** -0.5, Hq // Hkv
    want = [torch.zeros((Hkv, Lk, d), dtype=torch.float64, device=DEV) for _ in range(6)]  # dk, dv, their magnitudes, terms of dk
    for h in range(Hq):
        Q, K, V, dO, O = (x.double() for x in (q[0, h], k[0, h // G], v[0, h // G], do[0, h], out[0, h]))
        x = (Q @ K.T * scale).masked_fill(~M, -float("inf"))
        P = torch.softmax(x, 1)
        D = (dO * (P @ V)).sum(1, keepdim=True)
        dS = P * (dO @ V.T - D) * scale
        T = P * (dO.abs() @ V.abs().T + (dO * O).abs().sum(1, keepdim=True)) * scale
        close(dq[0, h], f64(dS @ K), f64(dS.abs() @ K.abs() + dS.abs().sum(1, keepdim=True) * (P @ K.abs())), dtype, f"dq of head {h}", f64(T @ K.abs()))
        for i, y in enumerate((dS.T @ Q, P.T @ dO, dS.abs().T @ Q.abs(), P.T @ dO.abs(), T.T @ Q.abs())):
            want[i][h // G] += y
    close(dk[0], f64(want[0]), f64(want[2]), dtype, "dk", f64(want[4]))
    close(dv[0], f64(want[1]), f64(want[3]), dtype, "dv")
    for x, y in zip((dq, dk, dv), usv.window_attn_backward(q, k, v, out, lse, do, **a)):
        assert torch.equal(x, y)


def test_empty_lengths(usv):
    q, k = torch.zeros((1, 2, 0, 64), device=DEV), torch.randn((1, 2, 5, 64), device=DEV)
    out, lse = usv.window_attn(q, k, k, -1, return_lse=True)
    assert out.shape == q.shape and lse.shape == (1, 2, 0)
    dq, dk, dv = usv.window_attn_backward(q, k, k, out, lse, q, -1)
    assert dq.shape == q.shape and not bool(dk.any()) and not bool(dv.any())
    out, lse = usv.window_attn(k, q, q, -1, return_lse=True)
    assert not bool(out.any()) and bool((lse == -float("inf")).all())
    dq, dk, dv = usv.window_attn_backward(k, q, q, out, lse, k, -1)
    assert not bool(dq.any()) and dk.shape == q.shape


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_logits_and_far_references(usv, dtype):
    """Logits of +-3e4 in either order of the keys, and rows whose logits all lie far below zero."""
    c = Case(1, 1, 1, 96, 96, 64, -1, -1)
    q, k, v, _ = inputs(c, TYPES[dtype], seed=40)
    ramp = torch.linspace(-1, 1, 96)[None, None, :, None]
    for sign in (1.0, -1.0):
        kk = (k.float() * 0 + sign * ramp * 180).to(TYPES[dtype])
        qq = (q.float() * 0 + torch.where(torch.arange(96) % 2 == 0, 20.0, -20.0)[None, None, :, None]).to(TYPES[dtype])
        ref, lse_ref, mag = wo.window_attn(f64(qq), f64(kk), f64(v), c.M)
        out, lse = usv.window_attn(qq.to(DEV), kk.to(DEV), v.to(DEV), -1, -1, return_lse=True)
        # a logit x carries 2^-24 of itself (times a few operations), which its weight sees whole
        slack = 8 * 2.0 ** -24 * 3e4
        bound = (slack + 1e-5 + (HALF_STEP if dtype == "bf16" else 0)) * mag + (HALF_STEP * np.abs(ref) if dtype == "bf16" else 0)
        assert (np.abs(f64(out) - ref) <= bound).all()
        close_lse(lse, lse_ref)


def test_same_call_same_bits(usv):
    """A call repeats its bits, forward and backward."""
    c = Case(3, 4, 2, 300, 300, 128, 100, 0, 5)
    q, k, v, do = (t.to(DEV) for t in inputs(c, torch.bfloat16, seed=50))
    run = lambda s: (lambda o: (*o, *usv.window_attn_backward(q[s], k[s], v[s], *o, do[s], **c.args)))(usv.window_attn(q[s], k[s], v[s], **c.args, return_lse=True))  # noqa: E731
    one = run(slice(0, 3))
    for x, y in zip(one, run(slice(0, 3))):
        assert torch.equal(x, y)


def test_workspace_of_few_rows(usv):
    """With and without scratch (shared out and in one piece) within the same bound; a workspace that is too small is refused."""
    c = Case(1, 2, 1, 5, 4000, 128, -1)
    q, k, v, _ = (t.to(DEV) for t in inputs(c, torch.bfloat16, seed=60))
    need = usv.window_workspace_bytes(q, k, -1)
    assert need > 0
    ref, lse_ref, mag = wo.window_attn(f64(q), f64(k), f64(v), c.M)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device=DEV)
    for w in (None, ws[:need], torch.empty(0, dtype=torch.uint8, device=DEV)):
        out, lse = usv.window_attn(q, k, v, -1, workspace=w, return_lse=True)
        close(out, ref, mag, "bf16", "out")
        close_lse(lse, lse_ref)
    assert bool((ws[need:] == 255).all())
    with pytest.raises(usv.UsvError) as e:
        usv.window_attn(q, k, v, -1, workspace=ws[: need - 16])
    assert e.value.status == 3


def test_graph_replays_and_streams(usv):
    """Forward and backward in one captured graph, replayed on new inputs with eager work between, against eager calls on another stream."""
    c = Case(2, 4, 2, 200, 200, 64, 50, 0, 3, 1, 0, [200, 77])
    args, lens = c.args, lens_of(c)
    st = [t.to(DEV) for t in inputs(c, torch.bfloat16, seed=70)]
    wsf = torch.empty(max(usv.window_workspace_bytes(st[0], st[1], **args), 16), dtype=torch.uint8, device=DEV)
    wsb = torch.empty(usv.window_workspace_bytes(st[0], st[1], **args, backward=True), dtype=torch.uint8, device=DEV)
    out, lse = torch.empty_like(st[0]), torch.empty(st[0].shape[:3], device=DEV)
    grads = [torch.empty_like(t) for t in st[:3]]

    def step():
        usv.window_attn(*st[:3], **args, q_start=0, seq_lens=lens, out=out, lse=lse, workspace=wsf)
        usv.window_attn_backward(*st[:3], out, lse, st[3], **args, q_start=0, seq_lens=lens, dq=grads[0], dk=grads[1], dv=grads[2], workspace=wsb)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    side = torch.cuda.Stream()
    for rep in range(4):
        new = [t.to(DEV) for t in inputs(c, torch.bfloat16, seed=80 + rep)]
        for dst, src in zip(st, new):
            dst.copy_(src)
        if rep == 2:
            lens.copy_(torch.tensor([13, 200], dtype=torch.int32))
            # (tokens that were padding hold NaN in these inputs: take ones without)
            for i, dst in enumerate(st):
                dst.copy_(normal(tuple(dst.shape), 90 + i, torch.bfloat16))
        for t in (out, lse, *grads):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            o, s = usv.window_attn(*st[:3], **args, q_start=0, seq_lens=lens, return_lse=True)
            g = usv.window_attn_backward(*st[:3], o, s, st[3], **args, q_start=0, seq_lens=lens)
        torch.cuda.current_stream().wait_stream(side)
        for x, y in zip((out, lse, *grads), (o, s, *g)):
            assert torch.equal(x, y), rep
        if rep == 2:
            lens.copy_(torch.tensor(c.lens, dtype=torch.int32))


def test_refusals(usv):
    q = torch.zeros((1, 4, 10, 64), dtype=torch.bfloat16, device=DEV)
    k = torch.zeros((1, 2, 12, 64), dtype=torch.bfloat16, device=DEV)
    f = usv.window_attn
    with pytest.raises(TypeError):
        f(q.cpu(), k, k, -1)
    with pytest.raises(TypeError):
        f(q, k.float(), k, -1)
    with pytest.raises(TypeError):
        f(q.half(), k.half(), k.half(), -1)
    with pytest.raises(ValueError):
        f(q, k, k[:, :, :11], -1)
    with pytest.raises(ValueError):
        f(q, k[:, :, :1].expand(1, 2, 12, 64), k, -1)
    with pytest.raises(ValueError):
        f(q, k, k, -1, seq_lens=torch.zeros(2, dtype=torch.int32, device=DEV))
    with pytest.raises(TypeError):
        f(q, k, k, -1, seq_lens=torch.zeros(1, dtype=torch.int64, device=DEV))
    with pytest.raises(ValueError):
        f(q, k, k, -1, out=q[:, :, :5])
    with pytest.raises(ValueError):
        f(q.transpose(2, 3).contiguous().transpose(2, 3), k, k, -1)
    for bad in (dict(left=-1, chunk=0), dict(left=-1, sinks=-1), dict(left=(1 << 30) + 1), dict(left=-1, q_start=-(1 << 30) - 1), dict(left=-1, scale=float("nan"))):
        with pytest.raises(usv.UsvError) as e:
            f(q, k, k, **bad)
        assert e.value.status == 1
    with pytest.raises(usv.UsvError) as e:
        f(q, torch.zeros((1, 3, 12, 64), dtype=torch.bfloat16, device=DEV), torch.zeros((1, 3, 12, 64), dtype=torch.bfloat16, device=DEV), -1)
    assert e.value.status == 1
    with pytest.raises(usv.UsvError) as e:
        f(q[..., :32], k[..., :32], k[..., :32], -1)
    assert e.value.status == 2
    x = torch.zeros((1, 4, 10, 68), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(usv.UsvError):  # rows that are not 16 bytes apart
        f(x[..., :64], k, k, -1)
    with pytest.raises(usv.UsvError):  # a start that is not 16-byte aligned
        f(torch.zeros((1, 4, 10, 72), dtype=torch.bfloat16, device=DEV)[..., 4:68], k, k, -1)
    with pytest.raises(usv.UsvError):  # an output whose rows overlap
        f(q, k, k, -1, out=torch.zeros((1, 1, 10, 64), dtype=torch.bfloat16, device=DEV).expand(1, 4, 10, 64))
    lse = torch.zeros((1, 4, 10), device=DEV)
    with pytest.raises(ValueError):
        usv.window_attn_backward(q, k, k, q, lse[:, :, :5].contiguous(), q, -1)
    with pytest.raises(usv.UsvError) as e:
        usv.window_attn_backward(q, k, k, q, lse, q, -1, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    assert e.value.status == 3
