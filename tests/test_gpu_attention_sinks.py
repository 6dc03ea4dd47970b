"""Attention where one key holds nearly all of the probability and its value is zero (a sink): what is left of the other keys has
to come out with the precision that keys of ordinary weight have, whatever format the probabilities take on their way."""
import numpy as np
import pytest
import torch

from oracle import glue
from test_gpu_paged import Attention, rd, status_clean  # noqa: F401

pytestmark = pytest.mark.gpu


def with_sink(rd, n, heads, kv, D, fmt, lens, at, bits, seed):  # noqa: F811
    """Channel 0 belongs to the sink: its key has 8 there, every other key 0, and the queries make that `bits` bits of weight."""
    a = Attention(rd, lens, [n] * len(lens), heads, kv, D, 16, fmt, seed=seed)
    ks = np.ones(kv) if a.ks is None else a.ks.astype(np.float64)
    vs = np.ones(kv) if a.vs is None else a.vs.astype(np.float64)
    q = glue.bf16_to_f32(a.qb).reshape(-1, heads, D).copy()
    q[..., 0] = (bits * np.log(2) / (8 * ks * a.scale)).repeat(heads // kv)
    a.qb = glue.f32_to_bf16(q.reshape(-1, heads * D))
    for b, length in enumerate(lens):
        ids = torch.from_numpy(a.table[b, :-(-length // 16)].astype(np.int64)).cuda()
        key = at % length
        for cache, store, sc, sink in ((a.kc, a.k, ks, True), (a.vc, a.v, vs, False)):
            x = cache[ids].float()                                  # [pages, kv, place, D]
            if sink:
                x[..., 0] = 0
                x[key // 16, :, key % 16, 0] = 8
            else:
                x[key // 16, :, key % 16] = 0
            cache[ids] = x.to(cache.dtype)
            store[b] = x.double().cpu().numpy().transpose(0, 2, 1, 3).reshape(-1, kv, D)[:length] * sc[None, :, None]
    return a


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("bits", [12, 20, 24])
@pytest.mark.parametrize("at", [0, 777, -1])
@pytest.mark.parametrize("n,heads,kv,D", [(1, 8, 2, 128), (5, 2, 1, 64), (9, 2, 2, 256), (20, 1, 1, 128), (40, 2, 2, 128), (70, 1, 1, 64), (33, 2, 1, 256)])
def test_attention_sink(rd, n, heads, kv, D, at, bits, fmt):  # noqa: F811
    """The bounds are those of ordinary keys (see Attention.check).  A key `bits` below the sink has a probability of about 2^-bits, the
    lowest of thousands some 2^-8 of that, where a 16-bit float that starts at 1 has no bits left."""
    a = with_sink(rd, n, heads, kv, D, fmt, [4000, 300, 1], at, bits, seed=n + bits)
    o, lse = a.run(False)
    a.check(o, lse, False)
    status_clean(rd)
