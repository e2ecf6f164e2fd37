"""CPU oracle (NumPy, 64 bits) of attention over a window with sinks, its gradient, and the quantised key/value cache.

Test infrastructure only, written from the definitions and sharing no code with the HIP path: the whole [queries, keys] truth matrix is
formed, hidden keys are left out of every sum, and the gradient is the softmax's derivative written out.
"""
from __future__ import annotations

import math

import numpy as np


def visible(q_pos, n, kv_len, left, right, sinks, chunk):
    """[len(q_pos), kv_len]: whether the query at a position sees the key at a position, in a sequence of n tokens."""
    p, j = np.asarray(q_pos, dtype=np.int64)[:, None], np.arange(kv_len, dtype=np.int64)[None, :]
    ok = (p >= 0) & (p < n) & (j < n)
    cp, cj = np.floor_divide(p, chunk), np.floor_divide(j, chunk)
    if right >= 0:
        ok = ok & (cj <= cp + right)
    if left >= 0:
        ok = ok & ((cj >= cp - left) | (cj < sinks))
    return ok


def masks(B, Lq, Lk, left, right, sinks, chunk, q_start=None, lens=None):
    """[B, Lq, Lk] truth values of a batch."""
    got = []
    for b in range(B):
        n = Lk if lens is None else min(max(int(lens[b]), 0), Lk)
        first = n - Lq if q_start is None else q_start
        got.append(visible(first + np.arange(Lq), n, Lk, left, right, sinks, chunk))
    return np.stack(got)


def _weights(q, k, M, scale):
    """P [queries, keys] and the log-sum-exp of one head; unseen keys' rows are not touched."""
    some = M.any(0)
    x = np.full(M.shape, -np.inf)
    live = M.any(1)
    if some.any():
        x[np.ix_(live, some)] = q[live] @ k[some].T * scale
    x = np.where(M, x, -np.inf)
    top = np.where(live, x.max(1, initial=-np.inf), 0.0)
    e = np.where(M, np.exp(x - top[:, None]), 0.0)
    l = e.sum(1)
    with np.errstate(divide="ignore"):
        return e / np.where(live, l, 1.0)[:, None], np.where(live, np.log(np.where(live, l, 1.0)) + top, -np.inf)


def window_attn(Q, K, V, M, scale=None):
    """Q [B, Hq, Lq, d], K, V [B, Hkv, Lk, d], M [B, Lq, Lk] -> out, lse, and sum_j P |v_j| (what relative errors of P act on)."""
    Q, K, V = (np.asarray(x, dtype=np.float64) for x in (Q, K, V))
    B, Hq, Lq, d = Q.shape
    G = Hq // K.shape[1]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    out, lse, mag = np.zeros(Q.shape), np.full((B, Hq, Lq), -np.inf), np.zeros(Q.shape)
    for b in range(B):
        some = M[b].any(0)
        for h in range(Hq):
            P, lse[b, h] = _weights(Q[b, h], K[b, h // G], M[b], scale)
            out[b, h] = P[:, some] @ V[b, h // G][some]
            mag[b, h] = P[:, some] @ np.abs(V[b, h // G][some])
    return out, lse, mag


def window_attn_backward(Q, K, V, dout, M, scale=None):
    """dq, dk, dv; for each what relative errors of P and dS act on; and what those of dout.v and D act on.  (In dq an error of a row's dS may
    be taken off all its keys in proportion to P, since dS adds up to 0: it then acts on sum P |k| too.)"""
    Q, K, V, dout = (np.asarray(x, dtype=np.float64) for x in (Q, K, V, dout))
    B, Hq, Lq, d = Q.shape
    G = Hq // K.shape[1]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    dq, dk, dv = np.zeros(Q.shape), np.zeros(K.shape), np.zeros(K.shape)
    mq, mk, mv = np.zeros(Q.shape), np.zeros(K.shape), np.zeros(K.shape)
    eq, ek = np.zeros(Q.shape), np.zeros(K.shape)
    for b in range(B):
        some, live = M[b].any(0), M[b].any(1)
        for h in range(Hq):
            g = h // G
            P = _weights(Q[b, h], K[b, g], M[b], scale)[0][np.ix_(live, some)]
            q, do, k, v = Q[b, h][live], dout[b, h][live], K[b, g][some], V[b, g][some]
            o = P @ v
            dS = P * (do @ v.T - (do * o).sum(1, keepdims=True)) * scale
            terms = P * (np.abs(do) @ np.abs(v).T + np.abs(do * o).sum(1, keepdims=True)) * scale  # sums of absolute products
            dq[b, h][live] = dS @ k
            dk[b, g][some] += dS.T @ q
            dv[b, g][some] += P.T @ do
            mq[b, h][live] = np.abs(dS) @ np.abs(k) + np.abs(dS).sum(1, keepdims=True) * (P @ np.abs(k))
            mk[b, g][some] += np.abs(dS).T @ np.abs(q)
            eq[b, h][live] = terms @ np.abs(k)
            ek[b, g][some] += terms.T @ np.abs(q)
            mv[b, g][some] += P.T @ np.abs(do)
    return (dq, dk, dv), (mq, mk, mv), (eq, ek, np.zeros(K.shape))


E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E4M3 = np.array([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:-1])  # (the last code is NaN)


def code_values(bits):
    """The value of every code of 4 or 8 bits."""
    if bits == 4:
        return np.concatenate([E2M1, -E2M1])
    one = np.append(E4M3, np.nan)
    return np.concatenate([one, -one])


def cache_values(X, bits):
    """What the cache holds of X [..., d]: per group of 32 channels the least scale 2^e at which the largest value lies no more than half a
    step beyond the largest code, and the nearest code (of two equally near ones the one of even number)."""
    X = np.asarray(X, dtype=np.float64)
    codes, border, least, last = (E2M1, 7.0, -125, 125) if bits == 4 else (E4M3, 464.0, -117, 119)
    g = X.reshape(-1, 32)
    out = np.full(g.shape, np.nan)
    for i, row in enumerate(g):
        if not np.isfinite(row).all():
            continue
        top = np.abs(row).max()
        e = least
        if top > 0:
            e = min(last, max(least, math.ceil(math.log2(top / border)) - 2))
            while top > border * 2.0 ** e and e < last:
                e += 1
        y = np.abs(row) / 2.0 ** e
        hi = np.clip(np.searchsorted(codes, y), 1, len(codes) - 1)
        lo = hi - 1
        near_hi = (codes[hi] - y < y - codes[lo]) | ((codes[hi] - y == y - codes[lo]) & (hi % 2 == 0))
        out[i] = np.copysign(np.where(near_hi, codes[hi], codes[lo]), row) * 2.0 ** e
    return out.reshape(X.shape)


def cache_decode(buf, page, row, head, which, page_size, d, bits):
    """The row of K (which 0) or V (1) that a cache buffer [pages, heads, bytes] holds at a place, from its bytes."""
    cb, sb = d * bits // 8, d // 32
    b = buf[page, head]
    codes = b[which * page_size * cb + row * cb:][:cb]
    scales = b[2 * page_size * cb + which * page_size * sb + row * sb:][:sb].astype(np.int64)
    if bits == 4:
        codes = np.stack([codes & 15, codes >> 4], -1).reshape(-1)
    x = code_values(bits)[codes].reshape(-1, 32) * 2.0 ** (scales[:, None] - 127.0)
    return np.where(scales[:, None] == 255, np.nan, x).reshape(-1)
