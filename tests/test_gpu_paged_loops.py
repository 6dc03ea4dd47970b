"""Sizes at which the loops of the paged-cache operators go round more than once: several passes of the query / key kernel per row,
several tiles per CTA and per cluster of the 4-bit products, cut items of later row tiles of attention; and queries whose
magnitude leaves f16."""
import numpy as np
import pytest
import torch

from helpers import bf16_to_np, to_dev_bf16
from oracle import glue, paged
from test_gpu_paged import U, Attention, cuda, e4m3_bits, qk_case, rd, status_clean  # noqa: F401

pytestmark = pytest.mark.gpu


# 32 / (D / 8) heads make a step, four steps a pass; with 5000 rows one warp works on a row (5 passes at 20 steps), with 2600 two
# (3 passes), with 1300 four (2 passes).  The last heads are values alone, in passes of their own with a low head count.
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("M,heads,kv,D,rot,pairs", [(5000, 24, 8, 128, 128, False), (2600, 24, 8, 128, 64, True), (1300, 24, 8, 128, 128, False), (5000, 12, 4, 256, 256, True),
                                                    (5000, 40, 20, 64, 32, False), (5000, 4, 24, 128, 0, False)])
def test_qk_rows_of_several_passes(rd, M, heads, kv, D, rot, pairs, fmt):  # noqa: F811
    rng, xb, w, cos, sin, pos = qk_case(M + D, M, heads, kv, D, rot)
    page, n_pages = 16, M // 16 + 3
    slots = rng.permutation(page * n_pages)[:M].astype(np.int64)
    slots[rng.random(M) < 0.1] = -1                                 # queries without an append
    pos[rng.random(M) < 0.1] = -1                                   # padding
    kind = torch.bfloat16 if fmt == "bf16" else torch.float8_e4m3fn
    k0, v0 = (torch.randn((n_pages, kv, page, D), device="cuda").to(kind) for _ in range(2))
    kc, vc = k0.clone(), v0.clone()
    scales = [np.exp(rng.standard_normal(kv) - 2).astype(np.float32) for _ in range(2)] if fmt == "e4m3" else [None, None]
    cache = rd.PagedCache(kc, vc, *(cuda(s) if s is not None else None for s in scales))
    Q = torch.full((M, heads * D), 3.0, dtype=torch.bfloat16, device="cuda")
    C, S = (cuda(cos), cuda(sin)) if rot else (None, None)
    rd.rudder_qk_norm_rope(rd.QkArgs(to_dev_bf16(xb), heads, kv, D, cuda(w[0]), cuda(w[1]), 1e-5, C, S, rd.ROPE_PAIRS if pairs else rd.ROPE_HALF, cuda(pos), Q, cache=cache,
                                     slots=cuda(slots)))
    q, k, v = paged.qk_norm_rope(glue.bf16_to_f32(xb), heads, kv, D, w[0], w[1], 1e-5, cos, sin, rot, pairs, pos)
    real = pos >= 0
    got = bf16_to_np(Q)
    assert np.array_equal(got[real], glue.f32_to_bf16(q.reshape(M, -1))[real])
    assert (got[~real] == glue.f32_to_bf16(np.full(1, 3.0, np.float32))[0]).all()
    put = np.flatnonzero(real & (slots >= 0))
    for have, start, rows, sc in ((kc, k0, k, scales[0]), (vc, v0, v, scales[1])):
        codes = glue.f32_to_bf16(rows) if fmt == "bf16" else e4m3_bits(rows, sc)
        bits = torch.int16 if fmt == "bf16" else torch.uint8
        want = start.view(bits).cpu().numpy().view(codes.dtype).copy()
        want[slots[put] // page, :, slots[put] % page] = codes[put]
        assert np.array_equal(have.view(bits).cpu().numpy().view(codes.dtype), want)
    status_clean(rd)


# One CTA for 16 channels: 300 and 321 tiles on 148 CTAs; a cluster of four for 64 channels: 75 and 76 tiles on 37 clusters.
@pytest.mark.parametrize("scheme,group", [("w4a8", 64), ("w4a8", 0), ("w4a4", 128), ("nvfp4", 16)])
@pytest.mark.parametrize("K,N,rows", [(512, 4800, (1, 5, 16)), (1024, 5120, (3, 8, 13)), (9216, 4800, (8, 16)), (9472, 4864, (1, 4, 7))])
def test_a16_several_tiles_per_cta(rd, scheme, group, K, N, rows):  # noqa: F811
    rng = np.random.default_rng(K + N)
    W = torch.from_numpy((rng.standard_normal((N, K)) * 0.02).astype(np.float32)).cuda()
    d = torch.from_numpy(np.exp(rng.uniform(-1.4, 1.4, K)).astype(np.float32)).cuda()
    w = rd.rudder_pack_weights(W, d, rd.SCHEMES[scheme], group or K)
    ex = {k: v.cpu() for k, v in rd.rudder_weight_export(w).items()}
    scales = ex["scales"].view(torch.float8_e4m3fn).float().numpy() if scheme == "nvfp4" else ex["scales"].float().numpy()
    ts = float(ex["tensor_scale"]) if scheme == "nvfp4" else None
    bias = rng.standard_normal(N).astype(np.float32)
    for M in rows:
        xb = glue.f32_to_bf16((rng.standard_normal((M, K)) * np.exp(rng.standard_normal((1, K)))).astype(np.float32))
        first = bf16_to_np(rd.rudder_linear_a16(w, to_dev_bf16(xb), cuda(bias)))
        y, s = paged.linear_a16(glue.bf16_to_f32(xb).astype(np.float64), ex["codes"].numpy(), scales, ex["dinv"].numpy(), bias, ts)
        got = glue.bf16_to_f32(first).astype(np.float64)
        assert (np.abs(got - y) <= 2.0 ** -8 * np.abs(y) + s * (2.0 ** -15 + K * 2 * U)).all(), (M, np.abs(got - y).max())
        for _ in range(3):                                          # the same bits again
            assert np.array_equal(bf16_to_np(rd.rudder_linear_a16(w, to_dev_bf16(xb), cuda(bias))), first)
    status_clean(rd)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("n,heads,kv,D", [(2, 4, 2, 128), (9, 2, 1, 64), (40, 2, 2, 128), (50, 1, 1, 256)])
@pytest.mark.parametrize("exponent", [60, -60, -100])
def test_attention_queries_far_from_one(rd, n, heads, kv, D, exponent, fmt):  # noqa: F811
    """The scale of the scores undoes the factor: a lost exponent or a flushed query shows at full size."""
    a = Attention(rd, [260, 1900], [n, n], heads, kv, D, 16, fmt, seed=n)
    q = glue.bf16_to_f32(a.qb).astype(np.float64)
    q[::3] *= 2.0 ** -7                                             # rows of a tile with ranges of their own
    a.qb = glue.f32_to_bf16((q * 2.0 ** exponent).astype(np.float32))
    a.scale = 0.1 * 2.0 ** -exponent
    for causal in (False, True):
        o, lse = a.run(causal)
        a.check(o, lse, causal)
    status_clean(rd)


# Row tiles are of 128 rows, so each of these has items of the second tile or a later one; the long contexts are cut over the CTAs and joined.
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lens,q_lens,heads,kv,D", [([9000], [150], 1, 1, 128), ([5000, 30], [100, 77], 2, 1, 64), ([4000, 700, 3], [50, 33, 40], 8, 1, 128), ([3000], [200], 2, 1, 256),
                                                    ([6000, 2000], [129, 257], 3, 1, 64), ([2500, 900], [90, 70], 8, 2, 128)])
def test_attention_later_row_tiles_cut_and_joined(rd, lens, q_lens, heads, kv, D, causal, fmt):  # noqa: F811
    a = Attention(rd, lens, q_lens, heads, kv, D, 32, fmt, seed=sum(q_lens), order="tokens")
    o, lse = a.run(causal, pad=3)
    a.check(o, lse, causal)
    o2, lse2 = a.run(causal, pad=3)
    assert np.array_equal(o, o2) and np.array_equal(lse, lse2)
    status_clean(rd)
