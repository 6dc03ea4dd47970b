"""Plain counterparts of the operators around the paged key-value cache, written from their definitions in numpy:
integers exactly, the bit-defined query / key pass in fp32 operation by operation, attention and the 4-bit products in fp64."""
from __future__ import annotations

import numpy as np

F = np.float32


def page_tables(old, new, free, table, page, capacity):
    """(table, slots, positions, starts, used): requests take pages of `free` in order."""
    table = table.copy()
    slots = np.full(capacity, -1, np.int64)
    positions = np.full(capacity, -1, np.int32)
    starts = np.zeros(len(old) + 1, np.int64)
    taken = 0
    t = 0
    for b, (o, n) in enumerate(zip(old.tolist(), new.tolist())):
        held, want = -(-o // page), -(-(o + n) // page)
        for c in range(held, want):
            if taken < len(free) and c < table.shape[1]:
                table[b, c] = free[taken]
            taken += 1
        first = taken - (want - held)
        for i in range(n):
            pos = o + i
            c = pos // page
            ok = c < table.shape[1] and (c < held or first + c - held < len(free))
            if t < capacity:
                positions[t] = pos
                if ok and table[b, c] >= 0:
                    slots[t] = int(table[b, c]) * page + pos % page
            t += 1
        starts[b + 1] = t
    return table, slots, positions, starts.astype(np.int32), taken


def head_norm(x, w, eps, rot=0, pairs=True):
    """RMS norm of [..., D] fp32 in the order of the kernel: lanes of 8 channels (both members of its half-split pairs in one lane), a lane's
    even and odd places on their own, the lanes combined by the exchange l ^ D/16, ..., 1."""
    D = x.shape[-1]
    place = np.arange(D).reshape(D // 8, 8)
    if rot and not pairs:
        for l in range(rot // 8):
            place[l] = np.concatenate([np.arange(4 * l, 4 * l + 4), rot // 2 + np.arange(4 * l, 4 * l + 4)])
    sq = (x * x).astype(F)[..., place]
    e, o = sq[..., 0], sq[..., 1]
    for i in range(1, 4):
        e, o = (e + sq[..., 2 * i]).astype(F), (o + sq[..., 2 * i + 1]).astype(F)
    s = (e + o).astype(F)
    d = D // 16
    lanes = np.arange(D // 8)
    while d:
        s = (s + s[..., lanes ^ d]).astype(F)
        d >>= 1
    mean = (s[..., :1] * F(1.0 / D)).astype(F)
    with np.errstate(divide="ignore", invalid="ignore"):
        r = (F(1) / np.sqrt((mean + F(eps)).astype(F)).astype(F)).astype(F)
        return ((x * r).astype(F) * w.astype(F)).astype(F)


def rotate(y, c, s, rot, pairs):
    """y [M, heads, D] fp32, c and s [M, rot / 2]: every product and sum rounded to fp32."""
    if rot == 0:
        return y
    y = y.copy()
    i = np.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if pairs else (i, i + rot // 2)
    c, s = c[:, None, :], s[:, None, :]
    u = ((y[..., a] * c).astype(F) - (y[..., b] * s).astype(F)).astype(F)
    v = ((y[..., b] * c).astype(F) + (y[..., a] * s).astype(F)).astype(F)
    y[..., a], y[..., b] = u, v
    return y


def qk_norm_rope(x, heads, kv_heads, D, qw, kw, eps, cos, sin, rot, pairs, positions):
    """x [M, (heads + 2 kv_heads) D] fp32 -> (q, k, v) fp32 [M, heads, D] before the rounding to the output type."""
    M = x.shape[0]
    x = x.reshape(M, heads + 2 * kv_heads, D).astype(F)
    q, k, v = x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]
    q, k = head_norm(q, qw, eps, rot, pairs), head_norm(k, kw, eps, rot, pairs)
    if rot:
        at = np.maximum(positions, 0)
        q, k = rotate(q, cos[at], sin[at], rot, pairs), rotate(k, cos[at], sin[at], rot, pairs)
    return q, k, v


def attention(q, k, v, scale, causal):
    """q [n, heads, D], k and v [L, kv_heads, D], fp64 -> (o, lse, a, ds): a = sum p |v| and ds = the largest sum of |q k| scale
    of each row, for error bounds."""
    n, heads, D = q.shape
    L, kv = k.shape[0], k.shape[1]
    g = heads // kv
    o = np.zeros((n, heads, D))
    a = np.zeros((n, heads, D))
    lse = np.full((n, heads), -np.inf)
    ds = np.zeros((n, heads))
    for h in range(heads):
        for t in range(n):
            see = max(0, min(L, L - n + t + 1)) if causal else L
            if see == 0:
                continue
            kk, vv = k[:see, h // g], v[:see, h // g]
            s = (kk @ q[t, h]) * scale
            m = s.max()
            p = np.exp(s - m)
            z = p.sum()
            o[t, h] = p @ vv / z
            a[t, h] = p @ np.abs(vv) / z
            lse[t, h] = m + np.log(z)
            ds[t, h] = (np.abs(kk) @ np.abs(q[t, h])).max() * abs(scale)
    return o, lse, a, ds


def linear_a16(x, codes, scales, dinv, bias, tensor_scale=None):
    """x [M, K] fp64; canonical codes uint8 [N, K/2], scales [N, groups] as numbers -> (y, s): s = sum |v w|, for error bounds."""
    N, K = codes.shape[0], codes.shape[1] * 2
    nib = np.empty((N, K), np.int64)
    nib[:, 0::2], nib[:, 1::2] = codes & 15, codes >> 4
    if tensor_scale is not None:
        grid = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
        w = np.where(nib >= 8, -1.0, 1.0) * grid[nib & 7] * float(tensor_scale)
    else:
        w = np.where(nib >= 8, nib - 16, nib).astype(np.float64)
    w = w * np.repeat(scales.astype(np.float64), K // scales.shape[1], axis=1)
    v = x * dinv.astype(np.float64)
    y, s = v @ w.T, np.abs(v) @ np.abs(w).T
    return (y + bias if bias is not None else y), s
