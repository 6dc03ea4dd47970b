"""rudder_attention_shared, on the GPU: values that are infinite or no numbers among the new tokens, and the precision of the probabilities."""
import numpy as np
import pytest
import torch

from helpers import bf16_to_np
from oracle import glue
from test_gpu_paged import rd, status_clean  # noqa: F401  (rd: the fixture)
from test_gpu_shared import Shared, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("prefix,own,n,heads,kv,D", [
    (320, [5, 40, 300], 3, 2, 2, 128), (1000, [9, 3000, 77], 9, 4, 2, 64), (129, [2500, 7, 20], 7, 6, 2, 256), (700, [20, 257, 64], 20, 1, 1, 64), (777, [70, 128, 1700], 70, 2, 2, 128),
    (333, [9000, 41], 40, 1, 1, 128), (64, [131, 33, 5000], 33, 2, 1, 256), (500, [5, 6, 60] * 12, 5, 8, 1, 64), (17, [4, 4], 4, 1, 1, 128), (0, [30, 300], 6, 2, 1, 64)])
def test_what_a_row_does_not_see_does_not_reach_it(rd, prefix, own, n, heads, kv, D, fmt):
    """Not a number or infinite among the new tokens' own keys and values: rows in front of that token keep their bits, rows that see it get it in its channels alone."""
    a = Shared(rd, [(prefix, [(t, n) for t in own])], heads, kv, D, 16, fmt, seed=n)
    lens = a.lens
    clean, lse = a.run_shared(True)
    a.check(clean, lse, True)
    clean, lse = clean.reshape(len(lens), n, heads, D), lse.reshape(len(lens), n, heads)
    if fmt == "bf16":
        bits, poison = torch.int16, [(float("nan"), 0x7FC0, "v"), (float("inf"), 0x7F80, "v"), (-float("inf"), 0xFF80 - 0x10000, "v"), (float("nan"), 0x7FC0, "k")]
    else:
        bits, poison = torch.uint8, [(float("nan"), 0x7F, "v"), (float("nan"), 0xFF, "k")]
    for back, (value, code, which) in zip((2, 1, n // 2, 3), poison):          # the key `back` before the end
        cache = (a.vc if which == "v" else a.kc).view(bits)
        saved = []
        for b, length in enumerate(lens):
            key = length - back
            pg, pl = int(a.table[b, key // 16]), key % 16
            saved.append((pg, pl, cache[pg, :, pl].clone()))
            cache[pg, :, pl, 0::2] = code
        o, l = a.run_shared(True)
        o, l = o.reshape(clean.shape), l.reshape(lse.shape)
        for b, length in enumerate(lens):
            for t in range(n):
                if length - back > length - n + t:                 # not seen
                    assert np.array_equal(o[b, t], clean[b, t]) and np.array_equal(l[b, t], lse[b, t]), (b, t, back)
                elif which == "k":
                    assert np.isnan(o[b, t]).all() and np.isnan(l[b, t]).all(), (b, t)
                else:
                    assert np.array_equal(o[b, t][:, 1::2], clean[b, t][:, 1::2]) and np.array_equal(l[b, t], lse[b, t]), (b, t)
                    even = o[b, t][:, 0::2]
                    assert (np.isnan(even) if np.isnan(value) else (even == value) | np.isnan(even)).all(), (b, t, back)
        for pg, pl, x in saved:
            cache[pg, :, pl] = x
    again, _ = a.run_shared(True)
    assert np.array_equal(again.reshape(clean.shape), clean)
    status_clean(rd)


def key_of(s):
    """Three bf16 numbers with s = k0 + k1 2^-8 + k2 2^-16 to 24 bits."""
    out = []
    for step in (1.0, 2.0 ** -8, 2.0 ** -16):
        k = torch.tensor(s / step, dtype=torch.float64).float().to(torch.bfloat16).item()
        out.append(k)
        s -= k * step
    return out


@pytest.mark.parametrize("B,n,D,own", [(10, 20, 128, False), (10, 20, 64, False), (2, 40, 128, False), (3, 70, 64, False), (2, 40, 256, False), (3, 40, 64, True), (3, 40, 128, True),
                                       (3, 40, 256, True)])
def test_probabilities_of_many_rows(rd, B, n, D, own):
    """A bf16 cache's probabilities enter as hi + lo, rounded to 2^-17: pairs of keys whose weighted values nearly cancel, with probabilities a little above 2^-1 whose hi is rounded
    down for the one and up for the other and whose lo is as long as it gets; in the prefix, or behind it.

    A score is a sum of three products that fp32 holds exactly (the pieces of a 24-bit number), times log2 e: exponent off by at most 3 x 2^-24, exp2 by 2^-22, so a
    probability by 2^-21 of itself.  Sums of 64 terms of fp32 accumulators: 2^-18 of the sum of magnitudes.  |o - o64| <= 2^-8 |o64| + a (2^-17 + 2^-21 + 2^-18), a = sum p |v|."""
    page, pairs = 64, 31
    rng = np.random.default_rng(D)
    s = np.zeros(64)
    for i in range(pairs):
        u = 0.5 * (1 + 2.0 ** -7 * rng.integers(0, 3))
        half = 2.0 ** -9                                           # half a step of a bf16 number in [0.5, 1)
        rest = half * (1 - 2.0 ** -8 * rng.uniform(0.03, 0.2))     # all places of lo are ones, and most of a step stands behind them
        s[2 * i], s[2 * i + 1] = np.log(u + rest), np.log(u + 2 * half - rest)
    k = np.zeros((64, D))
    for j in range(2 * pairs):
        k[j, :3] = key_of(s[j])
        s[j] = k[j, 0] + k[j, 1] * 2.0 ** -8 + k[j, 2] * 2.0 ** -16
    p = np.exp(s)
    v = np.zeros((64, D))
    for i in range(pairs):
        v[2 * i, i] = 1.0
        v[2 * i + 1, i] = -torch.tensor(p[2 * i] / p[2 * i + 1]).to(torch.bfloat16).item()
        left = p[2 * i] + p[2 * i + 1] * v[2 * i + 1, i]
        v[62, i] = -torch.tensor(left).to(torch.bfloat16).item()   # a key with probability one takes what is left
    # pages: 0 the tested keys, 1 keys of value zero; a request has both, the tested ones first or last
    kc, vc = torch.zeros((2 + B, 1, page, D)), torch.zeros((2 + B, 1, page, D))
    kc[0, 0], vc[0, 0] = torch.from_numpy(k).float(), torch.from_numpy(v).float()
    table = np.zeros((B, 2), np.int32)
    for b in range(B):
        table[b] = (1, 2 + b) if own else (0, 2 + b)
        if own:
            kc[2 + b], vc[2 + b] = kc[0], vc[0]
    cache = rd.PagedCache(kc.to(torch.bfloat16).cuda(), vc.to(torch.bfloat16).cuda())
    q = torch.zeros((B * n, D))
    q[:, 0], q[:, 1], q[:, 2] = 1.0, 2.0 ** -8, 2.0 ** -16
    O = torch.zeros((B * n, D), dtype=torch.bfloat16, device="cuda")
    attn = rd.AttentionArgs(q.to(torch.bfloat16).cuda(), 1, cache, i32(table), i32([128] * B), 1.0, O, max_q=n)
    rd.rudder_attention_shared(rd.SharedAttentionArgs(attn, i32([0, B]), i32([64]), i32([0]), B * n))
    got = glue.bf16_to_f32(bf16_to_np(O)).astype(np.float64)
    z = p.sum() + 64
    want, a = (p[:, None] * v).sum(0) / z, (p[:, None] * np.abs(v)).sum(0) / z
    bound = 2.0 ** -8 * np.abs(want) + a * (2.0 ** -17 + 2.0 ** -21 + 2.0 ** -18)
    assert (np.abs(got - want[None]) <= bound[None] + 1e-38).all(), (np.abs(got - want[None]) / (a + 1e-30)[None] * 2.0 ** 17).max()
    status_clean(rd)
