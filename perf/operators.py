"""Attention over a sliding window with sinks, its gradient, and the quantised cache that streaming generation reads, as cases for timing.

Five kinds of pass, each what one attention layer calls:

  window  window_attn: every query sees the chunks (frames; single tokens where chunk = 1) of a window around its own and the first
          `sinks` chunks
  grad    the layer of a training step: window_attn with its log-sum-exp, then window_attn_backward
  store   cache_write of the rows that a step has made, in 4 or 8 bits, and cache_read of the same rows
  fetch   cache_read of a long stretch of the cache
  decode  cache_attn: the newest tokens of every sequence attend to its cached keys and values

`own` false: the plain form, elementary torch operations in fp32.  `own` true: the framework's calls.

A cache is a tensor of bytes [pages, kv_heads, page_bytes]; per page and head it holds the K codes [page, d * bits / 8], the V codes,
the K scales [page, d / 32] and the V scales.  32 channels share a scale 2^(byte - 127); a code is e2m1 (two to a byte, the even channel
in the low half) or e4m3.  Inputs are N(0, 1) plus a vector that 64 consecutive tokens share, as neighbouring video tokens do.
"""
import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SLAB = 1 << 30  # logits of one step of the plain form (4 GiB in fp32): the large cases' whole matrices would not fit the card

FRAME_480P, FRAME_720P = 30 * 52, 45 * 80  # tokens of a latent frame


def listed():
    return [
        # the smallest call: one short clip's worth of tokens at d = 64, plain causal window with four sink tokens
        window("window_small", 1, 4, 4, 500, 500, 64, "bf16", 127, 0, 4, 1),
        # one layer of the 480p clip, frame by frame: a frame sees itself, the six before it and the first; straight from the projections
        window("window_480p_frames", 1, 12, 12, 21 * FRAME_480P, 21 * FRAME_480P, 128, "bf16", 6, 0, 1, FRAME_480P, packed=True),
        # 720p frames, both directions: three before and three after, the first stays visible: the largest call
        window("window_720p_frames", 1, 12, 12, 21 * FRAME_720P, 21 * FRAME_720P, 128, "bf16", 3, 3, 1, FRAME_720P),
        # token by token, shared key heads, a padded batch of ragged lengths
        window("window_tokens_gqa", 2, 32, 8, 8000, 8000, 128, "bf16", 4095, 0, 16, 1, ragged=True),
        # training steps: 480p frames; shared key heads at d = 64 in a padded batch; the fp32 accuracy path
        grad("grad_480p_frames", 1, 12, 12, 21 * FRAME_480P, 128, "bf16", 6, 0, 1, FRAME_480P),
        grad("grad_gqa_d64", 4, 16, 4, 2047, 64, "bf16", 511, 0, 8, 1, ragged=True),
        grad("grad_f32", 1, 2, 2, 4095, 128, "f32", 1023, 0, 16, 1),
        # what a generation step writes: one token for each of 32 sequences; three 480p frames
        {"name": "store_tokens", "kind": "store", "batch": 32, "kv_heads": 8, "rows": 1, "kv_len": 4096, "d": 128, "bits": 4, "page": 64, "dtype": "bf16"},
        {"name": "store_frames_8bit", "kind": "store", "batch": 1, "kv_heads": 12, "rows": 3 * FRAME_480P, "kv_len": 12 * FRAME_480P, "d": 128, "bits": 8, "page": 64, "dtype": "bf16"},
        # decoding one token for each of 64 sequences of ragged lengths
        decode("decode_batch", 64, 1, 32, 8, 32768, 128, 4, 64, -1, 0, 0, 1, ragged=True),
        # the next three 480p frames against the cached window and the first frame, 8 bits
        decode("decode_frames_8bit", 1, 3 * FRAME_480P, 12, 12, 12 * FRAME_480P, 128, 8, 64, 8, 0, 1, FRAME_480P),
        # a long stretch of the cache taken out for a layer that wants bf16
        {"name": "fetch_long", "kind": "fetch", "batch": 2, "kv_heads": 12, "rows": 9 * FRAME_480P + 7, "kv_len": 21 * FRAME_480P, "d": 128, "bits": 4, "page": 64, "dtype": "bf16"},
    ]


def window(name, batch, heads, kv_heads, q_len, kv_len, d, dtype, left, right, sinks, chunk, *, packed=False, ragged=False):
    return {"name": name, "kind": "window", "batch": batch, "heads": heads, "kv_heads": kv_heads, "q_len": q_len, "kv_len": kv_len, "d": d, "dtype": dtype,
            "left": left, "right": right, "sinks": sinks, "chunk": chunk, "packed": packed, "ragged": ragged}


def grad(name, batch, heads, kv_heads, tokens, d, dtype, left, right, sinks, chunk, *, ragged=False):
    return {**window(name, batch, heads, kv_heads, tokens, tokens, d, dtype, left, right, sinks, chunk, ragged=ragged), "kind": "grad"}


def decode(name, batch, q_len, heads, kv_heads, kv_len, d, bits, page, left, right, sinks, chunk, *, ragged=False):
    return {"name": name, "kind": "decode", "batch": batch, "heads": heads, "kv_heads": kv_heads, "q_len": q_len, "kv_len": kv_len, "d": d, "bits": bits, "page": page,
            "left": left, "right": right, "sinks": sinks, "chunk": chunk, "ragged": ragged}


def draw(rng):
    """One more case: kind by how often a model runs it, sizes over their whole ranges, odd ones among them."""
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = max(cost(c) for c in listed())
    while True:
        kind = rng.choice(["window", "window", "window", "grad", "grad", "decode", "decode", "decode", "store", "fetch"])
        kv_heads, group, d = spread(1, 12), rng.choice([1, 1, 2, 4, 8]), rng.choice([128, 128, 64])
        c = {"kind": kind, "batch": spread(1, 4), "d": d, "kv_heads": kv_heads}
        if kind in ("store", "fetch"):
            c["batch"] = spread(1, 32)
            c |= {"rows": spread(1, 20000), "bits": rng.choice([4, 4, 8]), "page": rng.choice([16, 32, 64, 64, 128, 240]), "dtype": rng.choice(["bf16", "bf16", "f32"])}
            c["kv_len"] = c["rows"] + spread(1, 8000)
        else:
            chunk = rng.choice([1, 1, 1, spread(16, 2000)])
            frames = rng.choice([-1, 0, 1, 2, 3, 7]) if chunk > 1 else rng.choice([-1, spread(1, 8000), spread(1, 8000)])
            c |= {"heads": kv_heads * group, "chunk": chunk, "left": frames, "sinks": rng.choice([0, 1]) if chunk > 1 else rng.choice([0, 0, 1, 4, spread(1, 200)]),
                  "right": rng.choice([0, 0, 0, 1]), "ragged": rng.choice([False, False, True])}
            if kind == "decode":
                c |= {"batch": spread(1, 64), "q_len": rng.choice([1, 1, 1, spread(2, 16), spread(16, 4000)]), "bits": rng.choice([4, 4, 8]), "page": rng.choice([16, 32, 64, 64, 128, 240])}
                c["kv_len"] = c["q_len"] + spread(1, 60000)
            else:
                n = spread(1, 33000) if kind == "window" else spread(1, 16000)
                c |= {"q_len": n, "kv_len": n, "dtype": rng.choice(["bf16", "bf16", "bf16", "f32"]), "packed": rng.choice([True, False])}
                if kind == "window" and rng.random() < 0.3:
                    c["kv_len"] = n + spread(1, 8000)  # the newest n tokens
        if cost(c) <= most and footprint(c) < 12e9:
            return c


# ---------------------------------------------------------------- sizes

def group_bytes(d, bits):
    """Bytes of one cached row (K or V of one head): codes and scales."""
    return d * bits // 8, d // 32


def lengths(case):
    """Valid tokens of each sequence."""
    B, n = case["batch"], case["kv_len"]
    return [max(1, n - (b * n) // (2 * B)) for b in range(B)] if case["ragged"] else [n] * B


def seen(case):
    """(pairs of query and key that see each other, keys that some query sees), summed over the batch, for one head."""
    import numpy as np

    pairs = keys = 0
    for n in lengths(case):
        first = (n if case["kind"] == "decode" else case["kv_len"]) - case["q_len"]
        p = np.arange(max(first, 0), min(first + case["q_len"], n), dtype=np.int64)
        if not p.size:
            continue
        c, T = p // case["chunk"], case["chunk"]
        hi = np.full_like(p, n) if case["right"] < 0 else np.minimum(n, (c + case["right"] + 1) * T)
        lo = np.zeros_like(p) if case["left"] < 0 else np.clip((c - case["left"]) * T, 0, None)
        s = np.minimum(case["sinks"] * T, hi)
        pairs += int((np.maximum(hi - np.maximum(lo, s), 0) + s).sum())
        first_key = max(int(lo[0]), int(s[-1]))
        keys += int(s[-1]) + max(0, int(hi[-1]) - first_key)
    return pairs, keys


def work(case):
    d, Hkv = case["d"], case["kv_heads"]
    if case["kind"] in ("store", "fetch"):
        rows = case["batch"] * Hkv * case["rows"] * 2
        e = 4 if case["dtype"] == "f32" else 2
        codes = sum(group_bytes(d, case["bits"]))
        return {"bytes": rows * (d * e + codes) * (2 if case["kind"] == "store" else 1), "flops": 0}
    pairs, keys = seen(case)
    H, rows = case["heads"], case["batch"] * case["q_len"]
    if case["kind"] == "decode":
        return {"bytes": 2 * keys * Hkv * sum(group_bytes(d, case["bits"])) + 2 * rows * H * d * 2, "flops": 4 * pairs * H * d}
    e = 4 if case["dtype"] == "f32" else 2
    once = rows * H * d * e * 2 + 2 * keys * Hkv * d * e
    if case["kind"] == "window":
        return {"bytes": once, "flops": 4 * pairs * H * d}
    # forward: q, k, v in, out; backward: those again with dout in, three gradients out
    return {"bytes": once + rows * H * d * e * 4 + 4 * keys * Hkv * d * e, "flops": 14 * pairs * H * d}


def cost(case):
    w = work(case)
    return w["flops"] * (8 if case.get("dtype") == "f32" else 1) / 1e15 + w["bytes"] / 5e12


def footprint(case):
    """Bytes that one state and the plain form of it take, roughly."""
    rows = case["batch"] * case["kv_heads"] * case["kv_len"] * case["d"]
    if case["kind"] in ("store", "fetch"):
        return 12 * rows
    q = case["batch"] * case["heads"] * case["q_len"] * case["d"]
    return 20 * rows + 20 * q + (12 * case["batch"] * case["heads"] * case["q_len"] * case["kv_len"] if case["kind"] == "decode" else 0)


# ---------------------------------------------------------------- inputs

def rng_of(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(shape, g, gain=1.0):
    """[B, H, L, d] in fp32: N(0, 1) plus `gain` times a vector that 64 consecutive tokens share."""
    x = torch.randn(shape, generator=g, device=DEV)
    shared = torch.randn((*shape[:2], -(-shape[2] // 64), shape[3]), generator=g, device=DEV)
    return x.add_(shared.repeat_interleave(64, dim=2)[:, :, : shape[2]], alpha=gain)


def tensor(B, H, L, d, dtype, g, packed=False, gain=1.0):
    x = normal((B, H, L, d), g, gain).to(dtype)
    return x.transpose(1, 2).contiguous().transpose(1, 2) if packed else x  # packed: as the projection [B, L, H, d] holds it


def prepare(case, seed):
    g = rng_of(seed)
    B, Hkv, d, kind = case["batch"], case["kv_heads"], case["d"], case["kind"]
    st = {"case": case}
    if kind in ("window", "grad"):
        dt, packed = DTYPES[case["dtype"]], case["packed"]
        st["q"] = tensor(B, case["heads"], case["q_len"], d, dt, g, packed)
        st["k"], st["v"] = (tensor(B, Hkv, case["kv_len"], d, dt, g, packed) for _ in range(2))
        st["lens"] = torch.tensor(lengths(case), dtype=torch.int32, device=DEV) if case["ragged"] else None
        if kind == "grad":
            st["dout"] = tensor(B, case["heads"], case["q_len"], d, dt, g, packed, gain=0.0)
        return st
    bits, page, n = case["bits"], case["page"], case["kv_len"]
    per = -(-n // page)  # pages of a sequence, anywhere in the cache
    st["table"] = torch.randperm(B * per, generator=g, device=DEV).to(torch.int32).reshape(B, per)
    st["cache"] = torch.zeros((B * per, Hkv, 2 * page * sum(group_bytes(d, bits))), dtype=torch.uint8, device=DEV)
    if kind == "store":
        st["k"], st["v"] = (tensor(B, Hkv, case["rows"], d, DTYPES[case["dtype"]], g, True) for _ in range(2))
        st["starts"] = torch.full((B,), n - case["rows"], dtype=torch.int32, device=DEV)
        return st
    for b in range(B):  # (one sequence at a time: the states of long caches are large)
        k, v = (normal((1, Hkv, n, d), g) for _ in range(2))
        put(st["cache"], k, v, st["table"][b: b + 1], torch.zeros(1, dtype=torch.int32, device=DEV), bits, page)
    if kind == "fetch":
        st["starts"] = torch.full((B,), n - case["rows"], dtype=torch.int32, device=DEV)
        return st
    st["lens"] = torch.tensor(lengths(case), dtype=torch.int32, device=DEV)
    st["q"] = tensor(B, case["heads"], case["q_len"], d, torch.bfloat16, g, True)
    return st


# ---------------------------------------------------------------- one pass

def run(st):
    return OWN[st["case"]["kind"]](st) if own else PLAIN[st["case"]["kind"]](st)


def usv():
    import paper_2512_05754_amd

    return paper_2512_05754_amd


def shape_args(c):
    return {"left": c["left"], "right": c["right"], "sinks": c["sinks"], "chunk": c["chunk"]}


def own_window(st):
    c = st["case"]
    return {"out": usv().window_attn(st["q"], st["k"], st["v"], **shape_args(c), seq_lens=st["lens"], q_start=c["kv_len"] - c["q_len"])}


def own_grad(st):
    c, u = st["case"], usv()
    out, lse = u.window_attn(st["q"], st["k"], st["v"], **shape_args(c), seq_lens=st["lens"], q_start=0, return_lse=True)
    dq, dk, dv = u.window_attn_backward(st["q"], st["k"], st["v"], out, lse, st["dout"], **shape_args(c), seq_lens=st["lens"], q_start=0)
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def own_store(st):
    c, u = st["case"], usv()
    u.cache_write(st["cache"], st["k"], st["v"], st["table"], st["starts"], bits=c["bits"])
    k, v = u.cache_read(st["cache"], st["table"], st["starts"], c["rows"], head_dim=c["d"], bits=c["bits"], dtype=DTYPES[c["dtype"]])
    return {"k": k, "v": v}


def own_fetch(st):
    c = st["case"]
    k, v = usv().cache_read(st["cache"], st["table"], st["starts"], c["rows"], head_dim=c["d"], bits=c["bits"], dtype=DTYPES[c["dtype"]])
    return {"k": k, "v": v}


def own_decode(st):
    c = st["case"]
    out, lse = usv().cache_attn(st["q"], st["cache"], st["table"], st["lens"], **shape_args(c), bits=c["bits"], return_lse=True)
    return {"out": out, "lse": lse}


OWN = {"window": own_window, "grad": own_grad, "store": own_store, "fetch": own_fetch, "decode": own_decode}


# ---- the plain forms

def visible(p, j, n, c):
    """[B, queries, keys] truth values: does the query at position p see the key at position j in a sequence of n tokens."""
    T = c["chunk"]
    cp, cj = torch.div(p, T, rounding_mode="floor")[:, :, None], torch.div(j, T, rounding_mode="floor")[:, None, :]
    ok = ((p >= 0) & (p < n))[:, :, None] & ((j >= 0) & (j < n))[:, None, :]
    if c["right"] >= 0:
        ok = ok & (cj <= cp + c["right"])
    if c["left"] >= 0:
        ok = ok & ((cj >= cp - c["left"]) | (cj < c["sinks"]))
    return ok


def slabs(st):
    """Query rows a, b whose logits fit, and the keys that they can see (sinks, then the window): one step where everything fits."""
    c = st["case"]
    n, T, first = c["kv_len"], c["chunk"], c["kv_len"] - c["q_len"]
    rows = max(1, SLAB // (c["batch"] * c["heads"] * n))
    if c["left"] >= 0:
        span = (c["left"] + c["right"] + c["sinks"] + 1) * T if c["right"] >= 0 else n
        rows = max(rows, min(4 * T if T > 1 else 1024, SLAB // (c["batch"] * c["heads"] * min(n, span + 1024))))
    for a in range(0, c["q_len"], rows):
        b = min(a + rows, c["q_len"])
        hi = n if c["right"] < 0 else min(n, ((first + b - 1) // T + c["right"] + 1) * T)
        lo = 0 if c["left"] < 0 else min(hi, max(0, ((first + a) // T - c["left"]) * T))
        s = min(c["sinks"] * T, lo)
        yield a, b, torch.cat([torch.arange(s, device=DEV), torch.arange(lo, hi, device=DEV)])


def logits(st, a, b, j):
    """Grouped queries a..b and their masked logits against the keys j: [B, kv_heads, group * rows, keys]."""
    c = st["case"]
    B, Hkv, d = c["batch"], c["kv_heads"], c["d"]
    G = c["heads"] // Hkv
    q = st["q"][:, :, a:b].float().reshape(B, Hkv, G * (b - a), d)
    k = st["k"][:, :, j].float()
    p = torch.arange(a, b, device=DEV) + (c["kv_len"] - c["q_len"])
    n = torch.full((B, 1), c["kv_len"], device=DEV) if st["lens"] is None else st["lens"][:, None].long()
    ok = visible(p.expand(B, -1), j.expand(B, -1), n, c)
    s = torch.matmul(q, k.transpose(2, 3)).mul_(1.0 / math.sqrt(d)).view(B, Hkv, G, b - a, -1)
    s.masked_fill_(~ok[:, None, None], -math.inf)
    return q, k, s.view(B, Hkv, G * (b - a), -1)


def softmax_of(s):
    """Weights (in place of s) and log-sum-exp of masked logits; a row without keys: zeros and -inf."""
    m = s.amax(-1, keepdim=True) if s.shape[-1] else torch.full((*s.shape[:-1], 1), -math.inf, device=s.device)
    m0 = torch.where(m == -math.inf, torch.zeros_like(m), m)
    e = s.sub_(m0).exp_()
    l = e.sum(-1, keepdim=True)
    lse = (l.log() + m0).squeeze(-1)
    return e.mul_(torch.where(l > 0, 1.0 / l, torch.zeros_like(l))), lse


def plain_window(st):
    c = st["case"]
    B, Hkv, d, H = c["batch"], c["kv_heads"], c["d"], c["heads"]
    out = torch.empty((B, H, c["q_len"], d), dtype=st["q"].dtype, device=DEV)
    for a, b, j in slabs(st):
        w = softmax_of(logits(st, a, b, j)[2])[0]
        out[:, :, a:b] = torch.matmul(w, st["v"][:, :, j].float()).view(B, H, b - a, d).to(out.dtype)
    return {"out": out}


def plain_grad(st):
    c = st["case"]
    B, Hkv, d, H, L = c["batch"], c["kv_heads"], c["d"], c["heads"], c["q_len"]
    dt = st["q"].dtype
    out, dq = (torch.empty((B, H, L, d), dtype=dt, device=DEV) for _ in range(2))
    lse = torch.empty((B, H, L), device=DEV)
    dk, dv = (torch.zeros((B, Hkv, c["kv_len"], d), device=DEV) for _ in range(2))
    scale = 1.0 / math.sqrt(d)
    for a, b, j in slabs(st):
        q, k, s = logits(st, a, b, j)
        w, ls = softmax_of(s)
        v = st["v"][:, :, j].float()
        o = torch.matmul(w, v)
        do = st["dout"][:, :, a:b].float().reshape(B, Hkv, -1, d)
        out[:, :, a:b], lse[:, :, a:b] = o.view(B, H, b - a, d).to(dt), ls.view(B, H, b - a)
        dv.index_add_(2, j, torch.matmul(w.transpose(2, 3), do))
        ds = torch.matmul(do, v.transpose(2, 3)).sub_((do * o).sum(-1, keepdim=True)).mul_(w).mul_(scale)
        dk.index_add_(2, j, torch.matmul(ds.transpose(2, 3), q))
        dq[:, :, a:b] = torch.matmul(ds, k).view(B, H, b - a, d).to(dt)
    return {"out": out, "lse": lse, "dq": dq, "dk": dk.to(dt), "dv": dv.to(dt)}


def regions(cache, page, d, bits):
    """K codes, V codes [pages, heads, page, d * bits / 8] and K scales, V scales [pages, heads, page, d / 32] of a cache, as views."""
    cb, sb = group_bytes(d, bits)
    at = [0, page * cb, 2 * page * cb, 2 * page * cb + page * sb, 2 * page * (cb + sb)]
    return [cache[:, :, x:y].unflatten(2, (page, -1)) for x, y in zip(at, at[1:])]


def places(table, pos, page):
    """Page and row in it of positions [B, n]."""
    return table.gather(1, torch.div(pos, page, rounding_mode="floor")).long(), pos % page


E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def power(e):
    """2^e in fp32 for whole e in -126..127."""
    return ((e + 127).int() << 23).view(torch.float32)


def quantise(x, bits):
    """Codes [..., d * bits / 8] and scale bytes [..., d / 32] of fp32 x [..., d]: the scale is the least power of two at which the largest
    value is no further than half a step beyond the largest code; codes are rounded to nearest, ties to even."""
    g = x.unflatten(-1, (-1, 32))
    m, e = torch.frexp(g.abs().amax(-1, keepdim=True))  # m in [0.5, 1)
    least, over, top = (-125, 0.875, 2) if bits == 4 else (-117, 0.90625, 8)
    e = torch.where(m == 0, least, (e - 1 - top + (m > over).int()).clamp_(min=least))
    y = (g * power(-e)).flatten(-2)
    if bits == 8:
        codes = y.clamp_(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        a = y.abs()
        h = (a > 0.25).to(torch.uint8)  # the borders between neighbouring codes; a tie goes to the even one
        for code, border in ((1, 0.75), (2, 1.25), (3, 1.75), (4, 2.5), (5, 3.5), (6, 5.0)):
            h += ((a >= border) if code % 2 else (a > border)).to(torch.uint8)
        h = h | (torch.signbit(y).to(torch.uint8) << 3)
        codes = h[..., 0::2] | (h[..., 1::2] << 4)
    return codes, (e.squeeze(-1) + 127).to(torch.uint8)


def put(cache, k, v, table, starts, bits, page):
    d = k.shape[-1]
    kc, vc, ks, vs = regions(cache, page, d, bits)
    pg, row = places(table, starts[:, None].long() + torch.arange(k.shape[2], device=DEV), page)
    for codes, scales, x in ((kc, ks, k), (vc, vs, v)):
        y, s = quantise(x.transpose(1, 2).float(), bits)
        codes[pg, :, row], scales[pg, :, row] = y, s


def values(codes, scales, bits):
    """fp32 [..., d] that codes [..., d * bits / 8] under scales [..., d / 32] stand for."""
    if bits == 8:
        x = codes.view(torch.float8_e4m3fn).float()
    else:
        of = torch.tensor([*E2M1, *(-e for e in E2M1)], device=DEV)
        x = of[torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()]
    return (x.unflatten(-1, (-1, 32)) * power(scales[..., None].int() - 127)).flatten(-2)


def take(st, pos):
    """K and V, fp32 [B, heads, n, d], at positions [B, n]."""
    c = st["case"]
    kc, vc, ks, vs = regions(st["cache"], c["page"], c["d"], c["bits"])
    pg, row = places(st["table"], pos, c["page"])
    return tuple(values(y[pg, :, row], s[pg, :, row], c["bits"]).transpose(1, 2) for y, s in ((kc, ks), (vc, vs)))


def plain_fetch(st):
    c = st["case"]
    k, v = take(st, st["starts"][:, None].long() + torch.arange(c["rows"], device=DEV))
    dt = DTYPES[c["dtype"]]
    return {"k": k.to(dt).contiguous(), "v": v.to(dt).contiguous()}


def plain_store(st):
    c = st["case"]
    put(st["cache"], st["k"], st["v"], st["table"], st["starts"], c["bits"], c["page"])
    return plain_fetch(st)


def plain_decode(st):
    c = st["case"]
    B, Hkv, d, H, L, T = c["batch"], c["kv_heads"], c["d"], c["heads"], c["q_len"], c["chunk"]
    n = st["lens"][:, None].long()
    most = c["kv_len"]
    p = n - L + torch.arange(L, device=DEV)
    j = torch.arange(most, device=DEV).expand(B, -1)
    if c["left"] >= 0:  # the sinks and a window's worth before the newest token
        s, span = min(c["sinks"] * T, most), min(most, (c["left"] + 1) * T + L)
        if s + span < most:
            j = torch.cat([torch.arange(s, device=DEV).expand(B, -1), (n - span) + torch.arange(span, device=DEV)], 1)
            j = torch.where((j < s) & (torch.arange(s + span, device=DEV) >= s), -1, j)  # the sinks once
    ok = visible(p, j, n, c)
    k, v = take(st, j.clamp(0, most - 1))
    G = H // Hkv
    q = st["q"].float().reshape(B, Hkv, G * L, d)
    w = torch.matmul(q, k.transpose(2, 3)).mul_(1.0 / math.sqrt(d)).view(B, Hkv, G, L, -1)
    w, lse = softmax_of(w.masked_fill_(~ok[:, None, None], -math.inf).view(B, Hkv, G * L, -1))
    return {"out": torch.matmul(w, v).view(B, H, L, d).to(torch.bfloat16), "lse": lse.view(B, H, L)}


PLAIN = {"window": plain_window, "grad": plain_grad, "store": plain_store, "fetch": plain_fetch, "decode": plain_decode}


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind in ("window", "grad"):
        got = exact_attention(case, st["q"], st["k"], st["v"], st.get("dout"), [case["kv_len"] - case["q_len"]] * case["batch"], lengths(case))
        return got if kind == "grad" else {"out": got["out"]}
    if kind == "store":
        dt = torch.float64
        return {n: exact_rounding(st[n].to(dt), case["bits"]) for n in ("k", "v")}
    if kind == "fetch":
        pos = [list(range(case["kv_len"] - case["rows"], case["kv_len"]))] * case["batch"]
        k, v = exact_rows(case, st, pos)
        return {"k": k, "v": v}
    lens = lengths(case)
    k, v = exact_rows(case, st, [range(case["kv_len"])] * case["batch"])
    return exact_attention(case, st["q"], k, v, None, [n - case["q_len"] for n in lens], lens)


def two_to(e):
    """2^e in 64 bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def exact_rounding(x, bits):
    """What the cache holds of x: the nearest multiple of the code's step, under the group's scale."""
    g = x.unflatten(-1, (-1, 32))
    top = g.abs().amax(-1, keepdim=True)
    largest, step_at_top = (6.0, 2.0) if bits == 4 else (448.0, 32.0)
    bound = largest + step_at_top / 2
    e = torch.ceil(torch.log2(torch.where(top > 0, top, torch.ones_like(top)) / bound))
    e = torch.where(top > two_to(e) * bound, e + 1, e)
    e = torch.where(top <= two_to(e - 1) * bound, e - 1, e)
    scale = two_to(e)
    y = g / scale
    binade = torch.floor(torch.log2(y.abs().clamp(min=1.0 if bits == 4 else 2.0 ** -6)))
    step = two_to(binade - (1 if bits == 4 else 3))
    return ((torch.round(y / step) * step).clamp(-largest, largest) * scale).flatten(-2)


def exact_rows(case, st, positions):
    d, bits, page = case["d"], case["bits"], case["page"]
    cb, sb = group_bytes(d, bits)
    if bits == 4:
        one = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
        of = torch.tensor(one + [-x for x in one], dtype=torch.float64, device=DEV)
    else:
        of = torch.tensor([(-1.0) ** (i >> 7) * ((i & 7) * 2.0 ** -9 if (i >> 3) & 15 == 0 else (8 + (i & 7)) * 2.0 ** (((i >> 3) & 15) - 10)) for i in range(256)],
                          dtype=torch.float64, device=DEV)
    got = [[], []]
    for b, pos in enumerate(positions):
        pos = torch.tensor(list(pos), device=DEV)
        row = pos % page
        pg = st["table"][b].long()[pos // page]
        for which in range(2):
            at = row * cb + which * page * cb
            heads = []
            for h in range(case["kv_heads"]):
                flat = st["cache"][:, h]
                y = flat[pg[:, None], at[:, None] + torch.arange(cb, device=DEV)].long()
                s = flat[pg[:, None], (2 * page * cb + which * page * sb + row * sb)[:, None] + torch.arange(sb, device=DEV)]
                if bits == 4:
                    y = torch.stack([y % 16, y // 16], -1).reshape(len(pos), d)
                heads.append(of[y] * two_to(s.long() - 127).repeat_interleave(32, dim=1))
            got[which].append(torch.stack(heads))
    return torch.stack(got[0]), torch.stack(got[1])


def exact_attention(case, q, k, v, dout, first, lens):
    """Sums over the keys that a query sees, in 64 bits; gradients from the softmax's derivative."""
    B, H, L, d = q.shape
    Hkv, N, T = k.shape[1], k.shape[2], case["chunk"]
    G, scale = H // Hkv, d ** -0.5
    dt = torch.float64
    out, lse = torch.zeros((B, H, L, d), dtype=dt, device=DEV), torch.full((B, H, L), -math.inf, dtype=dt, device=DEV)
    if dout is not None:
        dq, dk, dv = torch.zeros_like(out), torch.zeros((B, Hkv, N, d), dtype=dt, device=DEV), torch.zeros((B, Hkv, N, d), dtype=dt, device=DEV)
    rows = max(64, (1 << 27) // N)
    key = torch.arange(N, device=DEV)
    for b in range(B):
        for h in range(H):
            K, V = k[b, h // G].double(), v[b, h // G].double()
            for a in range(0, L, rows):
                z = min(L, a + rows)
                pos = torch.arange(a, z, device=DEV) + first[b]
                frame = torch.floor(pos.double() / T)[:, None]
                kf = torch.floor(key.double() / T)[None]
                hide = (pos < 0)[:, None] | (pos >= lens[b])[:, None] | (key >= lens[b])[None]
                if case["right"] >= 0:
                    hide = hide | (kf > frame + case["right"])
                if case["left"] >= 0:
                    hide = hide | ((kf < frame - case["left"]) & (kf >= case["sinks"]))
                some = torch.nonzero(~hide.all(0))[:, 0]
                if not len(some):
                    continue
                # only the keys that some row of the step sees: the rest weighs nothing
                hide, Ks, Vs = hide[:, some], K[some], V[some]
                Q = q[b, h, a:z].double()
                x = (Q @ Ks.T * scale).masked_fill(hide, -math.inf)
                ls = torch.logsumexp(x, 1)
                P = torch.exp(x - torch.where(torch.isinf(ls), 0.0, ls)[:, None])
                o = P @ Vs
                out[b, h, a:z], lse[b, h, a:z] = o, ls
                if dout is not None:
                    dO = dout[b, h, a:z].double()
                    dv[b, h // G].index_add_(0, some, P.T @ dO)
                    dS = P * (dO @ Vs.T - (dO * o).sum(1, keepdim=True)) * scale
                    dq[b, h, a:z] = dS @ Ks
                    dk[b, h // G].index_add_(0, some, dS.T @ Q)
    return {"out": out, "lse": lse} if dout is None else {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}
