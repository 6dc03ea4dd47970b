"""The operators around the paged key-value cache on the GPU, against their plain counterparts in the oracle (integers exactly, the
query / key pass bit for bit, attention and the 4-bit products in fp64).

Tolerances, derived before the first run (u = 2^-24, half a step of fp32; a bf16 rounding is off by at most 2^-8 of the value):
  attention  a score is a sum of D products in fp32 and one multiplication: off by at most ds (D + 4) 2u, ds = the row's largest
             sum |q k| scale; exp2 and the running rescaling add some 2^-21 per element.  Probabilities enter the second product with
             hi + lo bf16 (2^-16) or f16 (2^-11 with the subnormal end).  So |o - o64| <= 2^-8 |o64| + a (2 e_s + e_p + 2^-18),
             a = sum p |v|, e_s = ds (D + 4) 2u, e_p = 2^-15 or 2^-10; lse: e_s + 2^-20 (1 + |lse|) + n u.
  4-bit products   v enters with 16 bits (2^-16), fp32 sums of K terms: |y - y64| <= 2^-8 |y64| + s (2^-15 + K 2u), s = sum |v w|.
"""
import numpy as np
import pytest
import torch

import oracle
import workloads as wl
from helpers import GpuLinear, bf16_to_np, to_dev_bf16
from oracle import glue, paged

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def rd():
    import paper_2609_39056_b200 as rd
    rd.lib()
    return rd


def status_clean(rd):
    last, where = rd.rudder_device_status()
    assert last == 0, (last, where)


def cuda(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


# ---- page tables --------------------------------------------------------------------------------------------------------

def run_tables(rd, old, new, free, table, page, capacity):
    B = len(old)
    T = cuda(table.astype(np.int32))
    out = [torch.full((capacity,), 77, dtype=torch.int64, device="cuda"), torch.full((capacity,), 77, dtype=torch.int32, device="cuda"),
           torch.full((B + 1,), 77, dtype=torch.int32, device="cuda"), torch.full((1,), 77, dtype=torch.int32, device="cuda")]
    args = rd.PageTableArgs(cuda(old.astype(np.int32)), cuda(new.astype(np.int32)), cuda(free.astype(np.int32)), T, page, *out)
    rd.rudder_page_tables(args)
    first = [t.clone() for t in (T, *out)]
    rd.rudder_page_tables(args)                                    # the same inputs write the same again
    assert all(torch.equal(a, b) for a, b in zip(first, (T, *out)))
    return [t.cpu().numpy() for t in first]


@pytest.mark.parametrize("B,page,top,new_top", [(1, 16, 5, 1), (1, 1, 40, 40), (3, 8, 1, 1), (33, 64, 900, 200), (512, 16, 300, 1), (1025, 32, 200, 9),
                                                 (8192, 128, 700, 2)])
def test_page_tables(rd, B, page, top, new_top):
    rng = np.random.default_rng(B + page)
    old = rng.integers(0, top + 1, B)
    new = rng.integers(0, new_top + 1, B)
    old[rng.random(B) < 0.2] = 0
    new[rng.random(B) < 0.2] = 0
    held, want = -(-old // page), -(-(old + new) // page)
    width = int(want.max()) + 2
    ids = rng.permutation(int(want.sum()) + 7)
    table = np.full((B, width), -5, np.int32)
    at = 0
    for b in range(B):
        table[b, :held[b]] = ids[at:at + held[b]]
        at += held[b]
    capacity = int(new.sum()) + 5
    got = run_tables(rd, old, new, ids[at:], table, page, capacity)
    exp = paged.page_tables(old, new, ids[at:], table, page, capacity)
    for a, b in zip(got[:4], exp[:4]):
        assert np.array_equal(a, b)
    assert got[4][0] == exp[4]
    status_clean(rd)


def test_page_tables_exhausted_and_bad_lengths(rd):
    old, new = np.array([3, 0, 8]), np.array([2, 9, 1])
    table = np.full((3, 4), -1, np.int32)
    table[0, 0], table[2, :2] = 5, (6, 7)
    # 1 + 3 + 1 pages needed, 3 there: the tokens without a page get no slot
    free = np.array([10, 11, 12])
    got = run_tables(rd, old, new, free, table, 4, 12)
    exp = paged.page_tables(old, new, free, table, 4, 12)
    assert all(np.array_equal(a, b) for a, b in zip(got[:4], exp[:4])) and got[4][0] == 5
    assert rd.rudder_device_status() == (rd.ERR_ARG, rd.NO_PAGES)
    # the table is too narrow for request 1
    got = run_tables(rd, old, new, np.arange(20, 30), table[:, :2], 4, 12)
    exp = paged.page_tables(old, new, np.arange(20, 30), table[:, :2], 4, 12)
    assert all(np.array_equal(a, b) for a, b in zip(got[:4], exp[:4]))
    assert rd.rudder_device_status() == (rd.ERR_ARG, rd.NO_PAGES)
    # the slot map is too short
    got = run_tables(rd, old, new, np.arange(20, 30), table, 4, 7)
    exp = paged.page_tables(old, new, np.arange(20, 30), table, 4, 7)
    assert all(np.array_equal(a, b) for a, b in zip(got[:4], exp[:4]))
    assert rd.rudder_device_status() == (rd.ERR_ARG, rd.NO_ROOM)
    # lengths below zero count as zero; huge ones cannot wrap an index
    got = run_tables(rd, np.array([-4, 0]), np.array([2, -1]), np.array([3]), np.full((2, 2), -1), 4, 3)
    assert got[1].tolist() == [12, 13, -1] and got[3].tolist() == [0, 2, 2]
    assert rd.rudder_device_status() == (rd.ERR_ARG, rd.BAD_LENGTH)
    big = 2 ** 31 - 1
    got = run_tables(rd, np.array([big, 1, big]), np.array([big, 2, big]), np.array([3]), np.full((3, 2), -1), 4, 5)
    assert (got[1] == -1).all()
    assert rd.rudder_device_status()[0] == rd.ERR_ARG
    # a cached page that was never assigned
    got = run_tables(rd, np.array([1]), np.array([1]), np.array([3]), np.full((1, 2), -1), 4, 1)
    assert got[1].tolist() == [-1] and got[2].tolist() == [1]
    assert rd.rudder_device_status() == (rd.ERR_ARG, rd.BAD_PAGE)
    status_clean(rd)


# ---- query / key norm and rotation ----------------------------------------------------------------------------------------

def qk_case(seed, M, heads, kv, D, rot):
    rng = np.random.default_rng(seed)
    xb = glue.f32_to_bf16((rng.standard_normal((M, (heads + 2 * kv) * D)) * np.exp(rng.standard_normal((M, 1)))).astype(np.float32))
    w = [(1 + 0.2 * rng.standard_normal(D)).astype(np.float32) for _ in range(2)]
    n_pos = 97
    ang = rng.uniform(0, 6.3, (n_pos, max(rot // 2, 1)))
    pos = rng.integers(0, n_pos, M).astype(np.int32)
    return rng, xb, w, np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32), pos


def e4m3_bits(x, scale):
    """E4M3 codes of fp32 [M, kv, D] times the rounded reciprocal of the head's scale, saturating."""
    y = x * (np.float32(1) / scale.astype(np.float32))[None, :, None].astype(np.float32)
    return torch.from_numpy(np.clip(y, -448, 448)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()


QK_CASES = [(1, 1, 1, 64, 64), (7, 4, 4, 128, 128), (3, 3, 1, 256, 256), (130, 16, 2, 64, 32), (65, 5, 5, 128, 16), (9, 2, 1, 256, 48), (4, 24, 8, 128, 0),
            (300, 16, 16, 128, 128)]


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("M,heads,kv,D,rot", QK_CASES)
def test_qk_bit_exact_dense(rd, M, heads, kv, D, rot, pairs):
    rng, xb, w, cos, sin, pos = qk_case(M + D + rot, M, heads, kv, D, rot)
    if M > 4:
        xb[1] = 0                                                   # a row of zeros: eps decides
        pos[2] = -1                                                 # a row of padding
    q, k, _ = paged.qk_norm_rope(glue.bf16_to_f32(xb), heads, kv, D, w[0], w[1], 1e-6, cos, sin, rot, pairs, pos)
    X = to_dev_bf16(xb)
    wide_q = torch.full((M, heads * D + 24), 3.0, dtype=torch.bfloat16, device="cuda")
    wide_k = torch.full((M, kv * D + 8), 3.0, dtype=torch.bfloat16, device="cuda")
    style = rd.ROPE_PAIRS if pairs else rd.ROPE_HALF
    C, S = (cuda(cos), cuda(sin)) if rot else (None, None)
    args = rd.QkArgs(X, heads, kv, D, cuda(w[0]), cuda(w[1]), 1e-6, C, S, style, cuda(pos), wide_q[:, :heads * D], K=wide_k[:, 8:])
    rd.rudder_qk_norm_rope(args)
    want_q, want_k = glue.f32_to_bf16(q.reshape(M, -1)), glue.f32_to_bf16(k.reshape(M, -1))
    real = pos >= 0
    three = glue.f32_to_bf16(np.full(1, 3.0, np.float32))[0]
    got_q, got_k = bf16_to_np(wide_q), bf16_to_np(wide_k)
    assert np.array_equal(got_q[real][:, :heads * D], want_q[real]) and np.array_equal(got_k[real][:, 8:], want_k[real])
    assert (got_q[~real] == three).all() and (got_k[~real] == three).all() and (got_q[:, heads * D:] == three).all() and (got_k[:, :8] == three).all()
    # in place: queries and keys over themselves, values untouched
    Y = X.clone()
    args = rd.QkArgs(Y, heads, kv, D, cuda(w[0]), cuda(w[1]), 1e-6, C, S, style, cuda(pos), Y[:, :heads * D], K=Y[:, heads * D:(heads + kv) * D])
    rd.rudder_qk_norm_rope(args)
    got = bf16_to_np(Y)
    assert np.array_equal(got[real][:, :(heads + kv) * D], np.concatenate([want_q, want_k], 1)[real])
    assert np.array_equal(got[:, (heads + kv) * D:], xb[:, (heads + kv) * D:]) and np.array_equal(got[~real], xb[~real])
    status_clean(rd)


@pytest.mark.parametrize("order", ["heads", "tokens"])
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("M,heads,kv,D,rot", QK_CASES)
def test_qk_bit_exact_cache(rd, M, heads, kv, D, rot, fmt, order):
    rng, xb, w, cos, sin, pos = qk_case(M + D + rot + 1, M, heads, kv, D, rot)
    page, n_pages = (1, M + 3) if M < 4 else (16, M // 16 + 3)
    slots = rng.permutation(page * n_pages)[:M].astype(np.int64)
    if M > 4:
        pos[3], slots[4] = -1, -1                                   # padding; queries without an append
    kind = torch.bfloat16 if fmt == "bf16" else torch.float8_e4m3fn
    shape = (n_pages, kv, page, D) if order == "heads" else (n_pages, page, kv, D)
    k0, v0 = (torch.randn(shape, device="cuda").to(kind) for _ in range(2))
    kc, vc = k0.clone(), v0.clone()
    view = (lambda t: t) if order == "heads" else (lambda t: t.transpose(1, 2))
    scales = [np.exp(rng.standard_normal(kv) - 2).astype(np.float32) for _ in range(2)] if fmt == "e4m3" else [None, None]
    cache = rd.PagedCache(view(kc), view(vc), *(cuda(s) if s is not None else None for s in scales))
    Q = torch.full((M, heads * D), 3.0, dtype=torch.bfloat16, device="cuda")
    C, S = (cuda(cos), cuda(sin)) if rot else (None, None)
    args = rd.QkArgs(to_dev_bf16(xb), heads, kv, D, cuda(w[0]), cuda(w[1]), 1e-5, C, S, rd.ROPE_HALF, cuda(pos), Q, cache=cache, slots=cuda(slots))
    rd.rudder_qk_norm_rope(args)
    q, k, v = paged.qk_norm_rope(glue.bf16_to_f32(xb), heads, kv, D, w[0], w[1], 1e-5, cos, sin, rot, False, pos)
    real = pos >= 0
    assert np.array_equal(bf16_to_np(Q)[real], glue.f32_to_bf16(q.reshape(M, -1))[real])
    put = np.flatnonzero(real & (slots >= 0))
    for got, start, rows, sc in ((kc, k0, k, scales[0]), (vc, v0, v, scales[1])):
        codes = glue.f32_to_bf16(rows) if fmt == "bf16" else e4m3_bits(rows, sc)
        want = view(start).contiguous().view(torch.int16 if fmt == "bf16" else torch.uint8).cpu().numpy().view(codes.dtype).copy()
        want[slots[put] // page, :, slots[put] % page] = codes[put]
        have = view(got).contiguous().view(torch.int16 if fmt == "bf16" else torch.uint8).cpu().numpy().view(codes.dtype)
        assert np.array_equal(have, want)
    status_clean(rd)


def test_qk_defaults_and_bad_data(rd):
    M, D = 6, 64
    rng, xb, w, cos, sin, pos = qk_case(5, M, 2, 2, D, D)
    X = to_dev_bf16(xb)
    one = np.ones(D, np.float32)
    Q, K = (torch.zeros((M, 2 * D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rd.rudder_qk_norm_rope(rd.QkArgs(X, 2, 2, D, None, None, 0.0, None, None, rd.ROPE_HALF, None, Q, K=K))       # no weights, no rotation, no positions
    q, k, _ = paged.qk_norm_rope(glue.bf16_to_f32(xb), 2, 2, D, one, one, 0.0, None, None, 0, False, pos)
    assert np.array_equal(bf16_to_np(Q), glue.f32_to_bf16(q.reshape(M, -1))) and np.array_equal(bf16_to_np(K), glue.f32_to_bf16(k.reshape(M, -1)))
    status_clean(rd)
    # a position behind the tables: the row is skipped and recorded
    pos[1] = 97
    Q2 = torch.zeros_like(Q)
    rd.rudder_qk_norm_rope(rd.QkArgs(X, 2, 2, D, None, None, 0.0, cuda(cos), cuda(sin), rd.ROPE_HALF, cuda(pos), Q2, K=K))
    assert (Q2[1] == 0).all().item() and rd.rudder_device_status() == (rd.ERR_ARG, rd.BAD_POSITION)
    # a slot behind the cache: the queries are written, the append is skipped and recorded
    pos[1] = 0
    kc = torch.zeros((2, 2, 8, D), dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    slots = np.array([0, 16, 3, 2 ** 40, 7, 15])
    rd.rudder_qk_norm_rope(rd.QkArgs(X, 2, 2, D, None, None, 0.0, cuda(cos), cuda(sin), rd.ROPE_HALF, cuda(pos), Q2, cache=rd.PagedCache(kc, vc), slots=cuda(slots)))
    assert rd.rudder_device_status() == (rd.ERR_ARG, rd.BAD_SLOT)
    assert (Q2[1] != 0).any().item()
    written = (vc != 0).any(-1).any(1).cpu().numpy().reshape(-1)
    assert sorted(np.flatnonzero(written).tolist()) == [0, 3, 7, 15]
    status_clean(rd)


# ---- attention ------------------------------------------------------------------------------------------------------------

class Attention:
    """A cache with requests of the given lengths, and their queries."""

    def __init__(self, rd, lens, q_lens, heads, kv, D, page, fmt, seed=0, order="heads", spare=3, dead=float("nan"), far=None):
        rng = np.random.default_rng(seed)
        self.rd, self.lens, self.q_lens, self.heads, self.kv, self.D, self.page, self.fmt = rd, lens, q_lens, heads, kv, D, page, fmt
        pages = [-(-n // page) for n in lens]
        n_pages = sum(pages) + spare if far is None else far
        ids = rng.permutation(sum(pages) + spare) if far is None else n_pages - 1 - rng.permutation(sum(pages) + spare)
        width = max(1, max(pages)) + 1
        self.table = np.full((len(lens), width), -7, np.int32)
        kind = torch.bfloat16 if fmt == "bf16" else torch.float8_e4m3fn
        shape = (n_pages, kv, page, D) if order == "heads" else (n_pages, page, kv, D)
        k, v = (torch.empty(shape, dtype=kind, device="cuda") for _ in range(2))
        if far is None:
            for t in (k, v):
                t.copy_(torch.full(shape, dead, device="cuda").to(kind))      # what no request owns
        self.kc, self.vc = (k, v) if order == "heads" else (k.transpose(1, 2), v.transpose(1, 2))
        self.ks, self.vs = (None, None) if fmt == "bf16" else (np.exp(0.5 * rng.standard_normal(kv)).astype(np.float32) for _ in range(2))
        self.k, self.v = [], []
        at = 0
        for b, n in enumerate(lens):
            self.table[b, :pages[b]] = ids[at:at + pages[b]]
            at += pages[b]
            for store, cache, sc in ((self.k, self.kc, self.ks), (self.v, self.vc, self.vs)):
                x = torch.from_numpy(rng.standard_normal((n, kv, D)).astype(np.float32)).to(kind)
                store.append(x.to(torch.float64).numpy() * (1.0 if sc is None else sc.astype(np.float64)[None, :, None]))
                full = torch.full((pages[b] * page, kv, D), dead).to(kind)
                full[:n] = x
                cache[torch.from_numpy(self.table[b, :pages[b]].astype(np.int64)).cuda()] = full.view(pages[b], page, kv, D).transpose(1, 2).cuda()
        self.cache = rd.PagedCache(self.kc, self.vc, cuda(self.ks) if self.ks is not None else None, cuda(self.vs) if self.vs is not None else None)
        M = sum(q_lens)
        self.qb = glue.f32_to_bf16(rng.standard_normal((M, heads * D)).astype(np.float32))
        self.scale = 1.0 / np.sqrt(D)

    def run(self, causal, starts=True, pad=0, q_pad=0, stream=None):
        rd, M, width = self.rd, sum(self.q_lens), self.heads * self.D
        Q = torch.zeros((M + pad, width + q_pad), dtype=torch.bfloat16, device="cuda")
        Q[:M, :width] = to_dev_bf16(self.qb)
        O = torch.full((M + pad, width + 2 * q_pad), 5.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((M + pad, self.heads), 5.0, device="cuda")
        s = cuda(np.concatenate([[0], np.cumsum(self.q_lens)]).astype(np.int32)) if starts else None
        self.args = rd.AttentionArgs(Q[:, :width], self.heads, self.cache, cuda(self.table), cuda(np.array(self.lens, np.int32)), self.scale, O[:, :width], q_starts=s,
                                     max_q=max(1, max(self.q_lens)), causal=causal, lse=lse)
        rd.rudder_attention_paged(self.args, stream=stream)
        torch.cuda.synchronize()
        assert (O[M:] == 5.0).all().item() and (O[:, width:] == 5.0).all().item() and (lse[M:] == 5.0).all().item()
        self.O, self.lse = O, lse
        return glue.bf16_to_f32(bf16_to_np(O[:M, :width])).astype(np.float64).reshape(M, self.heads, self.D), lse[:M].cpu().numpy().astype(np.float64)

    def check(self, o, lse, causal):
        ep = 2.0 ** -15 if self.fmt == "bf16" else 2.0 ** -10
        q = glue.bf16_to_f32(self.qb).astype(np.float64).reshape(-1, self.heads, self.D)
        at = 0
        for b, n in enumerate(self.q_lens):
            wo, wl_, a, ds = paged.attention(q[at:at + n], self.k[b], self.v[b], self.scale, causal)
            es = ds * (self.D + 4) * 2 * U
            go, gl = o[at:at + n], lse[at:at + n]
            assert np.isfinite(go).all(), b
            assert (np.abs(go - wo) <= 2.0 ** -8 * np.abs(wo) + a * (2 * es[..., None] + ep + 2.0 ** -18) + 1e-38).all(), (b, np.abs(go - wo).max())
            empty = np.isneginf(wl_)
            assert np.array_equal(empty, np.isneginf(gl)), b
            w, g = wl_[~empty], gl[~empty]
            assert (np.abs(g - w) <= es[~empty] + 2.0 ** -20 * (1 + np.abs(w)) + self.lens[b] * U).all(), (b, np.abs(g - w).max())
            at += n


LENS = [0, 1, 2, 15, 16, 17, 31, 33, 64, 127, 129, 300, 511, 513]


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,kv,D,page", [(1, 1, 128, 16), (4, 4, 128, 8), (8, 1, 128, 64), (6, 2, 64, 16), (16, 1, 64, 32), (3, 3, 256, 16), (16, 2, 256, 128), (12, 1, 128, 1),
                                             (40, 2, 128, 256), (64, 1, 64, 16)])
def test_attention_one_token(rd, heads, kv, D, page, fmt):
    a = Attention(rd, LENS, [1] * len(LENS), heads, kv, D, page, fmt, seed=heads + D)
    o, lse = a.run(False, starts=False)
    a.check(o, lse, False)
    o2, lse2 = a.run(True, pad=3, q_pad=8)                         # one token sees all keys either way
    assert np.array_equal(o, o2) and np.array_equal(lse, lse2)
    status_clean(rd)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("q_lens,heads,kv,D", [([3, 1, 0, 5, 2], 4, 2, 128), ([7, 5, 1, 9, 4], 4, 4, 64), ([16, 0, 11, 2, 13], 2, 1, 128), ([40, 64, 1, 33, 20], 1, 1, 128),
                                               ([70, 3, 0, 129, 64], 2, 2, 64), ([5, 17, 2, 30, 8], 6, 2, 256)])
def test_attention_ragged_queries(rd, q_lens, heads, kv, D, causal, fmt):
    lens = [2, 700, 40, 133, 64]                                   # fewer keys than queries in places: rows that see nothing
    a = Attention(rd, lens, q_lens, heads, kv, D, 16, fmt, seed=D + heads)
    o, lse = a.run(causal, pad=2)
    a.check(o, lse, causal)
    status_clean(rd)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("lens,q,heads,kv,D,page", [([20011], 1, 2, 1, 128, 16), ([9000, 1, 13000], 1, 4, 1, 64, 32), ([5003], 64, 2, 2, 128, 64), ([6001, 77], 3, 8, 2, 256, 16),
                                                   ([4097] * 5, 20, 1, 1, 128, 128)])
def test_attention_long_is_split_and_joined(rd, lens, q, heads, kv, D, page, fmt):
    a = Attention(rd, lens, [q] * len(lens), heads, kv, D, page, fmt, seed=len(lens), order="tokens")
    o, lse = a.run(q > 1, starts=False)
    a.check(o, lse, q > 1)
    o2, lse2 = a.run(q > 1)                                        # the same bits again
    assert np.array_equal(o, o2) and np.array_equal(lse, lse2)
    status_clean(rd)


def test_attention_many_short_requests(rd):
    rng = np.random.default_rng(3)
    lens = rng.integers(0, 90, 700).tolist()
    a = Attention(rd, lens, [1] * 700, 2, 1, 64, 16, "bf16", seed=9)
    o, lse = a.run(False, starts=False)
    a.check(o, lse, False)
    status_clean(rd)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("T,heads,kv,D", [(20, 2, 2, 64), (33, 1, 1, 128), (70, 2, 2, 128), (9, 4, 2, 256), (130, 1, 1, 64)])
def test_attention_many_short_requests_of_many_rows(rd, T, heads, kv, D, fmt):
    """Items of one tile each, most with warps that own no row: nothing may run ahead of the item that is being written out."""
    rng = np.random.default_rng(T)
    n = 500 if T < 70 else 160
    lens = rng.integers(0, 140, n).tolist()
    q_lens = rng.integers(1, T + 1, n).tolist()
    a = Attention(rd, lens, q_lens, heads, kv, D, 16, fmt, seed=T)
    first = None
    for _ in range(5):
        o, lse = a.run(False)
        status_clean(rd)
        assert first is None or (np.array_equal(o, first[0]) and np.array_equal(lse, first[1]))
        first = (o, lse)
    a.check(o, lse, False)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_attention_large_scores_and_small_queries(rd, fmt):
    a = Attention(rd, [260, 77], [2, 2], 4, 2, 128, 16, fmt, seed=2)
    for factor in (200.0, 2.0 ** -60, 2.0 ** -126):               # one key takes all; queries far below the range of f16
        a.qb = glue.f32_to_bf16((glue.bf16_to_f32(a.qb) * np.float32(factor)).astype(np.float32))
        a.scale = 0.5
        o, lse = a.run(False)
        a.check(o, lse, False)
    status_clean(rd)


def test_attention_far_pages(rd):
    """A cache of 5.6 GB per tensor: pages behind 2^31 elements and 2^32 bytes."""
    page, kv, D = 64, 8, 128
    n_pages = (int(2.8e9) // (page * kv * D)) + 1
    a = Attention(rd, [333, 64, 1], [1, 2, 1], 8, kv, D, page, "bf16", seed=4, far=n_pages)
    assert int(a.table[0, 0]) * page * kv * D > 2 ** 31
    o, lse = a.run(False)
    a.check(o, lse, False)
    # and the append at the far end
    x = torch.randn((2, 3 * kv * D), device="cuda").to(torch.bfloat16)
    Q = torch.empty((2, kv * D), dtype=torch.bfloat16, device="cuda")
    slots = torch.tensor([n_pages * page - 1, n_pages * page - 70], device="cuda")
    rd.rudder_qk_norm_rope(rd.QkArgs(x, kv, kv, D, None, None, 1e-6, None, None, rd.ROPE_HALF, None, Q, cache=a.cache, slots=slots))
    assert torch.equal(a.vc[n_pages - 1, :, page - 1].reshape(-1), x[0, 2 * kv * D:]) and torch.equal(a.vc[n_pages - 2, :, page - 6].reshape(-1), x[1, 2 * kv * D:])
    status_clean(rd)


def test_attention_bad_data_is_recorded(rd):
    a = Attention(rd, [40, 40, 40], [1, 1, 1], 2, 1, 64, 16, "bf16", seed=6, dead=0.0)
    good, _ = a.run(False)
    keep = a.table.copy()
    for bad in (-1, 2 ** 30):
        a.table = keep.copy()
        a.table[1, 1] = bad
        o, _ = a.run(False)
        assert rd.rudder_device_status() == (rd.ERR_ARG, rd.BAD_PAGE)
        assert np.array_equal(o[[0, 2]], good[[0, 2]]) and np.isfinite(o).all()
    a.table = keep
    lens = a.lens
    for bad in (-3, 2 ** 31 - 1):
        a.lens = [40, bad, 40]
        o, _ = a.run(False)
        assert rd.rudder_device_status()[0] == rd.ERR_ARG
        assert np.array_equal(o[[0, 2]], good[[0, 2]])
    a.lens = lens
    # row ranges that leave Q, fall back, or are longer than max_q: nothing outside is touched
    a.run(False)
    args = a.args
    for starts in ([0, 1, 2, 9], [0, 2, 1, 3], [-5, 1, 2, 3], [0, 3, 3, 3]):
        args.keep[4].copy_(torch.tensor(starts, dtype=torch.int32))
        rd.rudder_attention_paged(args)
        assert rd.rudder_device_status() == (rd.ERR_ARG, rd.BAD_LENGTH)
    status_clean(rd)


def test_attention_output_over_queries(rd):
    a = Attention(rd, [3000, 5], [4, 4], 4, 2, 128, 32, "bf16", seed=12)
    want, _ = a.run(False)
    Q = to_dev_bf16(a.qb)
    args = rd.AttentionArgs(Q, 4, a.cache, cuda(a.table), cuda(np.array(a.lens, np.int32)), a.scale, Q, max_q=4)
    rd.rudder_attention_paged(args)
    assert np.array_equal(glue.bf16_to_f32(bf16_to_np(Q)).reshape(8, 4, 128), want)


# ---- 4-bit products of a few rows -------------------------------------------------------------------------------------------

A16 = [("w4a8", 64), ("w4a8", 128), ("w4a8", 0), ("w4a4", 64), ("w4a4", 128), ("w4a4", 0), ("nvfp4", 16)]


@pytest.mark.parametrize("K,N", [(256, 64), (768, 320), (2048, 2048), (4608, 192), (8192, 128), (14336, 64), (18432, 64)])
@pytest.mark.parametrize("scheme,group", A16)
def test_linear_a16(rd, scheme, group, K, N):
    rng = np.random.default_rng(K + N)
    W = torch.from_numpy((rng.standard_normal((N, K)) * 0.02).astype(np.float32)).cuda()
    W[3] = 0
    d = torch.from_numpy(np.exp(rng.uniform(-1.4, 1.4, K)).astype(np.float32)).cuda()
    w = rd.rudder_pack_weights(W, d, rd.SCHEMES[scheme], group or K)
    ex = {k: v.cpu() for k, v in rd.rudder_weight_export(w).items()}
    scales = ex["scales"].view(torch.float8_e4m3fn).float().numpy() if scheme == "nvfp4" else ex["scales"].float().numpy()
    ts = float(ex["tensor_scale"]) if scheme == "nvfp4" else None
    bias = rng.standard_normal(N).astype(np.float32)
    for M in (1, 2, 4, 5, 8, 9, 16):
        xb = glue.f32_to_bf16((rng.standard_normal((M, K)) * np.exp(rng.standard_normal((1, K)))).astype(np.float32))
        wide = torch.zeros((M, K + 8), dtype=torch.bfloat16, device="cuda")
        wide[:, :K] = to_dev_bf16(xb)
        out = torch.full((M, N + 16), 3.0, dtype=torch.bfloat16, device="cuda")
        b = bias if M % 2 else None
        rd.rudder_linear_a16(w, wide[:, :K], cuda(b) if b is not None else None, out[:, :N])
        y, s = paged.linear_a16(glue.bf16_to_f32(xb).astype(np.float64), ex["codes"].numpy(), scales, ex["dinv"].numpy(), b, ts)
        got = glue.bf16_to_f32(bf16_to_np(out[:, :N])).astype(np.float64)
        assert (np.abs(got - y) <= 2.0 ** -8 * np.abs(y) + s * (2.0 ** -15 + K * 2 * U)).all(), (M, np.abs(got - y).max())
        assert (out[:, N:] == 3.0).all().item()
    status_clean(rd)


def test_linear_a16_refusals(rd):
    w = rd.rudder_pack_weights(torch.randn(64, 128, device="cuda"), None, rd.W4A8_INT, 64)
    x = torch.randn((17, 128), device="cuda").to(torch.bfloat16)
    y = torch.zeros((17, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(rd.RudderError) as e:
        rd.rudder_linear_a16(w, x, None, y)
    assert e.value.status == rd.ERR_SHAPE
    L, h = rd.lib(), w.handle
    p, o = x.data_ptr(), y.data_ptr()
    assert L.rudder_linear_a16(h, p, 128, 0, None, o, 64, None) == rd.ERR_SHAPE
    assert L.rudder_linear_a16(h, None, 128, 1, None, o, 64, None) == rd.ERR_ARG
    for bad in ((p + 2, 128, None, o, 64), (p, 120, None, o, 64), (p, 132, None, o, 64), (p, 128, None, o + 8, 64), (p, 128, None, o, 56), (p, 128, p + 4, o, 64)):
        assert L.rudder_linear_a16(h, bad[0], bad[1], 1, bad[2], bad[3], bad[4], None) == rd.ERR_ALIGN
    assert (y == 0).all().item()
    wide = rd.rudder_pack_weights(torch.randn(64, 36864 + 128, device="cuda"), None, rd.W4A8_INT, 64)
    with pytest.raises(rd.RudderError) as e:
        rd.rudder_linear_a16(wide, torch.zeros((1, wide.K), dtype=torch.bfloat16, device="cuda"))
    assert e.value.status == rd.ERR_SHAPE


def test_arguments_on_another_device_are_refused(rd):
    a = Attention(rd, [5], [1], 1, 1, 64, 16, "bf16")
    with pytest.raises(rd.RudderError):
        rd.AttentionArgs(to_dev_bf16(a.qb), 1, a.cache, torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 1.0, to_dev_bf16(a.qb))


# ---- attention: more of what the calls allow ---------------------------------------------------------------------------------

@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("lens,n,heads,kv,D", [([40, 3, 333], 5, 2, 2, 128), ([3000], 9, 4, 2, 64), ([130, 2500], 7, 6, 2, 256), ([50, 257, 4, 64], 20, 1, 1, 64),
                                               ([128, 90, 1700], 70, 2, 2, 128), ([9000], 40, 1, 1, 128), ([131, 3, 5000], 33, 2, 1, 256)])
def test_attention_what_a_row_does_not_see_does_not_reach_it(rd, lens, n, heads, kv, D, fmt):
    """Not a number or infinite among the new tokens' own keys and values: the rows in front of that token keep their bits."""
    a = Attention(rd, lens, [n] * len(lens), heads, kv, D, 16, fmt, seed=n)
    clean, lse = a.run(True)
    a.check(clean, lse, True)

    def at(b, key):                                                # page and place of a key
        return int(a.table[b, key // 16]), key % 16
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
            if key >= 0:
                pg, pl = at(b, key)
                saved.append((b, pg, pl, cache[pg, :, pl].clone()))
                cache[pg, :, pl, 0::2] = code
        o, l = a.run(True)
        o, l = o.reshape(clean.shape), l.reshape(lse.shape)
        for b, length in enumerate(lens):
            for t in range(n):
                if not 0 <= length - back <= length - n + t:       # not seen (or not there)
                    assert np.array_equal(o[b, t], clean[b, t]) and np.array_equal(l[b, t], lse[b, t]), (b, t, back)
                elif which == "k":
                    assert np.isnan(o[b, t]).all() and np.isnan(l[b, t]).all(), (b, t)
                else:
                    assert np.array_equal(o[b, t][:, 1::2], clean[b, t][:, 1::2]) and np.array_equal(l[b, t], lse[b, t]), (b, t)
                    even = o[b, t][:, 0::2]
                    assert (np.isnan(even) if np.isnan(value) else even == value).all(), (b, t, back)
        for b, pg, pl, x in saved:
            cache[pg, :, pl] = x
    again, _ = a.run(True)
    assert np.array_equal(again.reshape(clean.shape), clean)
    status_clean(rd)


@pytest.mark.parametrize("order", ["heads", "tokens"])
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("page", [1, 2, 4, 8, 32, 64, 128, 1024])
@pytest.mark.parametrize("n,heads,kv,D", [(40, 2, 2, 128), (9, 4, 1, 64), (33, 2, 2, 256), (3, 4, 2, 128)])
def test_attention_page_sizes_and_orders(rd, n, heads, kv, D, page, fmt, order):
    lens = [700, 129, 5, 2049]
    a = Attention(rd, lens, [n] * 4, heads, kv, D, page, fmt, seed=page, order=order)
    o, lse = a.run(True, pad=1, q_pad=8)
    a.check(o, lse, True)
    status_clean(rd)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("n,heads,kv,D", [(1, 2, 2, 128), (5, 4, 2, 64), (50, 2, 2, 128), (40, 1, 1, 256)])
@pytest.mark.parametrize("scale", [-0.31, 0.0])
def test_attention_scales_of_any_sign(rd, n, heads, kv, D, scale, fmt):
    a = Attention(rd, [300, 17, 2000, n // 2], [n] * 4, heads, kv, D, 16, fmt, seed=n)
    a.scale = scale
    for causal in (False, True):
        o, lse = a.run(causal)
        a.check(o, lse, causal)
    status_clean(rd)


@pytest.mark.parametrize("n", [1, 6, 40])
@pytest.mark.parametrize("B", [31, 32, 33, 100])
def test_attention_request_counts(rd, B, n):
    """Up to 32 requests are placed by each warp alone, more of them by the whole CTA; long ones are cut either way."""
    rng = np.random.default_rng(B + n)
    lens = rng.integers(0, 2500, B).tolist()
    q_lens = rng.integers(0, n + 1, B).tolist()
    q_lens[0] = n
    a = Attention(rd, lens, q_lens, 2, 1, 64, 32, "bf16", seed=B)
    o, lse = a.run(True, pad=2)
    a.check(o, lse, True)
    # nothing to do at all: no keys, then no queries
    a.lens = [0] * B
    o, lse = a.run(False)
    assert (o == 0).all() and np.isneginf(lse).all()
    _, _, kv_lens, O, q_starts, _ = a.args.keep
    kv_lens.copy_(torch.tensor(lens, dtype=torch.int32))
    q_starts.fill_(0)
    O.fill_(3.0)
    rd.rudder_attention_paged(a.args)
    assert (O == 3.0).all().item()
    status_clean(rd)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("n,D", [(40, 128), (20, 256), (64, 64)])
def test_attention_bad_pages_under_many_rows(rd, n, D, fmt):
    a = Attention(rd, [400, 400, 400], [n] * 3, 2, 1, D, 16, fmt, seed=6, dead=0.0)
    good, _ = a.run(False)
    keep = a.table.copy()
    for where in (3, 24):                                          # in a whole tile, in the request's last one
        for bad in (-1, 2 ** 30, a.kc.shape[0]):
            a.table = keep.copy()
            a.table[1, where] = bad
            o, _ = a.run(False)
            assert rd.rudder_device_status() == (rd.ERR_ARG, rd.BAD_PAGE)
            assert np.array_equal(o[:n], good[:n]) and np.array_equal(o[2 * n:], good[2 * n:]) and np.isfinite(o).all()
    a.table = keep
    o, _ = a.run(False)
    assert np.array_equal(o, good)
    status_clean(rd)


def test_attention_far_pages_under_many_rows(rd):
    page, kv, D = 64, 8, 128
    n_pages = (int(2.8e9) // (page * kv * D)) + 1
    a = Attention(rd, [333, 64, 1], [40, 33, 1], 8, kv, D, page, "bf16", seed=4, far=n_pages)
    o, lse = a.run(True)
    a.check(o, lse, True)
    status_clean(rd)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("n,heads,kv,D", [(1, 8, 2, 128), (40, 2, 2, 128)])
def test_attention_captured_follows_the_lengths(rd, n, heads, kv, D, fmt):
    """A captured call replayed with other lengths and tables, over its own queries: the device's data decide."""
    a = Attention(rd, [3000, 70, 500], [n] * 3, heads, kv, D, 16, fmt, seed=5)
    want, _ = a.run(True)
    a.lens = [1200, 64, 1]
    want2, _ = a.run(True)
    a.lens = [3000, 70, 500]
    lens = cuda(np.array(a.lens, np.int32))
    Q = to_dev_bf16(a.qb)
    X = Q.clone()
    args = rd.AttentionArgs(X, heads, a.cache, cuda(a.table), lens, a.scale, X, max_q=n, causal=True)
    rd.rudder_attention_paged(args)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rd.rudder_attention_paged(args)
    for L, w in (([3000, 70, 500], want), ([1200, 64, 1], want2), ([3000, 70, 500], want)):
        lens.copy_(torch.tensor(L, dtype=torch.int32))
        X.copy_(Q)
        graph.replay()
        assert np.array_equal(glue.bf16_to_f32(bf16_to_np(X)).reshape(w.shape), w)
    status_clean(rd)
