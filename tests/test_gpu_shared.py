"""The operators for many requests that continue one context, on the GPU, against their plain counterparts in the oracle: pages exactly, attention with a
shared prefix and low-rank adapters in fp64.

Tolerances, derived before the first run (u = 2^-24, half a step of fp32; a bf16 rounding is off by at most 2^-8 of the value):
  attention  as in test_gpu_paged.py; joining the prefix's part to a row's own is one more rescaling of each (2^-21, inside its e_p).
  adapters   the inner sum is off by at most K 2u of the sum of its products' magnitudes and enters the outer one with 2^-16 of itself, the outer sum
             has R terms, twice (hi and lo): |y - y64| <= 2^-8 |y64| + s (2^-16 + (K + 2 R + 16) 2u), s = |base| + |scale| sum |b| sum |a x|.
"""
import numpy as np
import pytest
import torch

from helpers import bf16_to_np, to_dev_bf16
from oracle import glue, paged, shared
from test_gpu_paged import Attention, U, cuda, rd, status_clean  # noqa: F401  (rd: the fixture)

pytestmark = pytest.mark.gpu


def i32(v):
    return torch.tensor(np.asarray(v, np.int32), device="cuda")


# ---- pages ------------------------------------------------------------------------------------------------------------------

def layers(rd, n, n_pages, heads, page, D, fmt, order="heads", seed=0):
    """n caches of random bytes (every bit pattern, NaN among them) and their PagedCaches."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, word = (torch.bfloat16, torch.int16) if fmt == "bf16" else (torch.float8_e4m3fn, torch.uint8)
    shape = (n_pages, heads, page, D) if order == "heads" else (n_pages, page, heads, D)
    out = []
    for _ in range(2 * n):
        lo, hi = (-32768, 32768) if word == torch.int16 else (0, 256)
        t = torch.randint(lo, hi, shape, generator=g, device="cuda").to(word).view(kind)
        out.append(t if order == "heads" else t.transpose(1, 2))
    return out, rd.PagedCaches([rd.PagedCache(out[i], out[i + 1]) for i in range(0, 2 * n, 2)])


def words(t):
    return t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.uint8).cpu().numpy()


def pool(rng, B, page, top, share=0.5, spare=5, cols=None):
    """(table, lens, pages of the pool): requests that share beginnings, on pages all over the pool."""
    lens = rng.integers(0, top + 1, B)
    pages = -(-lens // page)
    width = cols or max(1, pages.max()) + 1
    n_pages = int(pages.sum()) + spare
    ids = rng.permutation(n_pages)
    table = np.full((B, width), -5, np.int32)
    at = 0
    for b in range(B):
        table[b, :pages[b]] = ids[at:at + pages[b]]
        at += pages[b]
        if b and rng.random() < share:
            s = min(lens[b], lens[b - 1]) // page
            table[b, :s] = table[b - 1, :s]
    return table, lens.astype(np.int32), n_pages


def run_fork(rd, table, lens, page, src, dst, free, fork_lens, taken, caches):
    T, L = i32(table), i32(lens)
    copies, used = torch.full((len(src), 3), 77, dtype=torch.int32, device="cuda"), i32([77])
    args = rd.PageForkArgs(T, L, page, i32(src), i32(dst), i32(free), used, fork_lens=None if fork_lens is None else i32(fork_lens),
                           taken=None if taken is None else i32([taken]), copies=copies)
    rd.rudder_page_fork(args, caches)
    first = [t.clone() for t in (T, L, copies, used)]
    rd.rudder_page_fork(args, caches)                              # the same inputs write the same again
    assert all(torch.equal(a, b) for a, b in zip(first, (T, L, copies, used)))
    return [t.cpu().numpy() for t in first]


@pytest.mark.parametrize("parents,n,page,top,n_layers,heads,D,fmt,order", [
    (1, 1, 16, 5, 1, 1, 64, "bf16", "heads"), (1, 8, 16, 333, 2, 4, 128, "bf16", "heads"), (3, 7, 1, 40, 1, 2, 64, "e4m3", "heads"), (5, 64, 64, 700, 9, 3, 128, "e4m3", "tokens"),
    (2, 33, 8, 90, 8, 1, 256, "bf16", "tokens"), (4, 600, 32, 200, 1, 2, 64, "bf16", "heads"), (700, 1300, 16, 60, 1, 1, 64, "e4m3", "heads"), (2, 3, 1024, 3000, 1, 2, 64, "e4m3", "heads"),
    (2, 5, 256, 1000, 3, 2, 256, "bf16", "heads")])
@pytest.mark.parametrize("cut", [False, True])
def test_fork(rd, parents, n, page, top, n_layers, heads, D, fmt, order, cut):
    rng = np.random.default_rng(n + page)
    table, lens, n_pages = pool(rng, parents, page, top, spare=n + 4)
    lens[0] = top
    table, lens, n_pages = table, lens, n_pages
    if -(-top // page) > (table[0] >= 0).sum():                    # (the longest request's pages)
        extra = -(-top // page)
        wide = np.full((parents, max(table.shape[1], extra + 1)), -5, np.int32)
        wide[:, :table.shape[1]] = table
        wide[0, :extra] = n_pages + np.arange(extra)
        table, n_pages = wide, n_pages + extra
    free = np.setdiff1d(np.arange(n_pages), table)[::-1].copy()
    full = np.concatenate([table, np.full((n, table.shape[1]), -5, np.int32)])
    order_of_rows = rng.permutation(parents + n)                   # parents and children lie in any order
    T = np.empty_like(full)
    T[order_of_rows] = full
    L = np.empty(parents + n, np.int32)
    L[order_of_rows] = np.concatenate([lens, rng.integers(0, 99, n)])
    src = order_of_rows[rng.integers(0, parents, n)]
    dst = order_of_rows[parents:]
    fork_lens = (L[src] * rng.random(n)).astype(np.int32) if cut else None
    caches, handle = layers(rd, n_layers, n_pages, heads, page, D, fmt, order, seed=n)
    before = [words(c) for c in caches]
    want = shared.fork(T, L, page, src.tolist(), dst.tolist(), free, fork_lens, 2 if cut else 0)
    got = run_fork(rd, T, L, page, src, dst, free, fork_lens, 2 if cut else None, handle)
    for g, w in zip(got, want):
        assert np.array_equal(g.reshape(np.shape(w)), w)
    assert (want[1][dst] >= 0).all()
    for c, b in zip(caches, before):
        assert np.array_equal(words(c), shared.copy_tokens(b, want[2]))
    status_clean(rd)


def test_fork_without_caches_and_lists(rd):
    T, L, used = i32([[4, 5, -1], [-1, -1, -1]]), i32([20, 0]), i32([9])
    rd.rudder_page_fork(rd.PageForkArgs(T, L, 16, i32([0]), i32([1]), i32([3]), used))
    assert T.tolist() == [[4, 5, -1], [4, 3, -1]] and L.tolist() == [20, 20] and used.tolist() == [1]
    status_clean(rd)


def test_fork_leaves_out_what_cannot_be(rd):
    rng = np.random.default_rng(5)
    table, lens, n_pages = pool(rng, 9, 8, 60, share=0, spare=4)
    lens[:4] = [13, 16, 21, 40]
    table, lens, n_pages = np.where(np.arange(12)[None] < 8, np.arange(9 * 12).reshape(9, 12) % 72, -1).astype(np.int32), lens, 90
    free = [80, 81, -1, 95, 84, 85]
    cases = [([0, 0, 2], [4, 4, 5], None, free, rd.BAD_LENGTH),             # a row taken twice: the first has it
             ([0, 2], [2, 5], None, free, rd.BAD_LENGTH),                   # a row that another child reads
             ([0, 9, -1], [5, 6, 7], None, free, rd.BAD_LENGTH), ([0, 2], [9, -1], None, free, rd.BAD_LENGTH),
             ([0, 2, 2], [5, 6, 7], [14, -1, 20], free, rd.BAD_LENGTH),     # longer than the parent, below zero
             ([0, 2, 0, 1], [4, 5, 6, 7], None, free, rd.NO_PAGES),         # the third has no page; the fourth needs none
             ([0, 2], [4, 5], None, [80], rd.NO_PAGES), ([0, 2], [4, 5], None, [80, 99], rd.BAD_PAGE), ([0], [4], None, [], rd.NO_PAGES)]
    for src, dst, fork_lens, fr, code in cases:
        caches, handle = layers(rd, 2, n_pages, 2, 8, 64, "bf16", seed=3)
        before = [words(c) for c in caches]
        want = shared.fork(table, lens, 8, src, dst, fr, fork_lens, 0, n_pages)
        got = run_fork(rd, table, lens, 8, src, dst, np.array(fr, np.int32), fork_lens, None, handle)
        assert rd.rudder_device_status() == (rd.ERR_ARG, code), (src, dst)
        for g, w in zip(got, want):
            assert np.array_equal(g.reshape(np.shape(w)), w), (src, dst)
        for c, b in zip(caches, before):
            assert np.array_equal(words(c), shared.copy_tokens(b, want[2]))
    # a parent's page that is none: the child has its page, nothing is copied, and it is recorded
    bad = table.copy()
    bad[0, 1] = 1000
    caches, handle = layers(rd, 1, n_pages, 2, 8, 64, "bf16", seed=3)
    before = [words(c) for c in caches]
    run_fork(rd, bad, lens, 8, [0], [4], np.array(free, np.int32), None, None, handle)
    assert rd.rudder_device_status() == (rd.ERR_ARG, rd.BAD_PAGE)
    assert all(np.array_equal(words(c), b) for c, b in zip(caches, before))
    # the list begins behind what is taken, which may be all of it
    got = run_fork(rd, table, lens, 8, [0], [4], np.array(free, np.int32), None, 100, handle)
    assert rd.rudder_device_status() == (rd.ERR_ARG, rd.NO_PAGES) and got[1][4] == lens[4]


@pytest.mark.parametrize("n_layers,heads,page,D,fmt,order", [(1, 1, 1, 64, "e4m3", "heads"), (3, 5, 16, 128, "bf16", "tokens"), (12, 2, 64, 256, "e4m3", "heads"), (128, 1, 8, 64, "bf16", "heads")])
def test_copy(rd, n_layers, heads, page, D, fmt, order):
    rng = np.random.default_rng(page)
    n_pages, n = 61, 30
    ids = rng.permutation(n_pages)
    copies = np.stack([ids[:n], ids[n:2 * n], rng.integers(0, page + 1, n)], 1).astype(np.int32)
    copies[3, 0], copies[5, 1] = -1, -1                            # entries that are none
    for count in (None, 17, 0):
        caches, handle = layers(rd, n_layers, n_pages, heads, page, D, fmt, order, seed=n)
        before = [words(c) for c in caches]
        rd.rudder_page_copy(rd.PageCopyArgs(i32(copies), None if count is None else i32([count])), handle)
        for c, b in zip(caches, before):
            assert np.array_equal(words(c), shared.copy_tokens(b, copies[:count]))
        status_clean(rd)


def test_copy_bad_entries_are_recorded(rd):
    caches, handle = layers(rd, 1, 9, 2, 8, 64, "bf16")
    before = words(caches[0])
    for entry, code in (([9, 1, 2], rd.BAD_PAGE), ([1, 9, 2], rd.BAD_PAGE), ([1, 2, 9], rd.BAD_LENGTH), ([1, 2, -1], rd.BAD_LENGTH)):
        rd.rudder_page_copy(rd.PageCopyArgs(i32([entry, [3, 3, 8]])), handle)
        assert rd.rudder_device_status() == (rd.ERR_ARG, code)
    assert np.array_equal(words(caches[0]), before)
    rd.rudder_page_copy(rd.PageCopyArgs(i32([[0, 1, 4]]), i32([2])), handle)
    assert rd.rudder_device_status() == (rd.ERR_ARG, rd.BAD_LENGTH)
    assert np.array_equal(words(caches[0]), shared.copy_tokens(before, [(0, 1, 4)]))


POOLS = [(1, 16, 5, 0), (1, 1, 1, 0), (9, 16, 349, 40), (33, 8, 300, 3), (512, 64, 2000, 11), (300, 1, 400, 9000), (3, 32, 40000, 2), (2000, 16, 20, 70000)]


@pytest.mark.parametrize("B,page,top,spare", POOLS)
@pytest.mark.parametrize("drop", [0.0, 0.4, 1.0])
def test_release(rd, B, page, top, spare, drop):
    rng = np.random.default_rng(B + page)
    table, lens, n_pages = pool(rng, B, page, top, spare=max(1, spare))
    gone = rng.permutation(B)[:int(drop * B)]
    gone = np.concatenate([gone, gone[:2]])                        # the same request twice is once
    T, L = i32(table), i32(lens)
    refs, free, n_free = (torch.full((n,), 77, dtype=torch.int32, device="cuda") for n in (n_pages, n_pages, 1))
    args = rd.PageReleaseArgs(T, L, page, refs, free, n_free, drop=i32(gone) if len(gone) else None)
    for _ in range(2):
        rd.rudder_page_release(args)
        want = shared.release(table, lens, page, gone, n_pages)
        for g, w in zip((L, refs, free, n_free), want):
            assert np.array_equal(g.cpu().numpy().reshape(np.shape(w)), w)
    assert np.array_equal(T.cpu().numpy(), table)
    status_clean(rd)


@pytest.mark.parametrize("B,page,top,spare", POOLS)
@pytest.mark.parametrize("in_place", [False, True])
def test_compact_plan(rd, B, page, top, spare, in_place):
    rng = np.random.default_rng(B + page + 1)
    table, lens, n_pages = pool(rng, B, page, top, spare=max(1, spare))
    lens[rng.permutation(B)[:B // 3]] = 0
    want = shared.compact(table, lens, page, n_pages)
    T, L = i32(table), i32(lens)
    N = T if in_place else torch.full_like(T, 77)
    remap, copies, n_copies, n_live = (torch.full(s, 77, dtype=torch.int32, device="cuda") for s in ((n_pages,), (n_pages // 2, 3), (1,), (1,)))
    rd.rudder_page_compact(rd.PageCompactArgs(T, L, page, N, remap, copies, n_copies, n_live))
    m = len(want[2])
    assert n_copies.tolist() == [m] and n_live.tolist() == [want[3]]
    assert np.array_equal(N.cpu().numpy(), want[0]) and np.array_equal(remap.cpu().numpy(), want[1])
    assert np.array_equal(copies[:m].cpu().numpy(), want[2]) and (copies[m:] == 77).all().item()
    status_clean(rd)


@pytest.mark.parametrize("n_layers,heads,D,fmt,order", [(1, 3, 64, "bf16", "heads"), (9, 1, 128, "e4m3", "tokens")])
def test_compact_moves_the_pages(rd, n_layers, heads, D, fmt, order):
    """What every request reads through its table stays the same, and nothing is held above n_live any more."""
    rng = np.random.default_rng(3)
    page = 16
    table, lens, n_pages = pool(rng, 20, page, 700, spare=200)
    lens[::3] = 0
    caches, handle = layers(rd, n_layers, n_pages, heads, page, D, fmt, order)
    before = [words(c) for c in caches]
    T = i32(table)
    remap, copies, n_copies, n_live = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((n_pages,), (n_pages // 2, 3), (1,), (1,)))
    rd.rudder_page_compact(rd.PageCompactArgs(T, i32(lens), page, T, remap, copies, n_copies, n_live), handle)
    new = T.cpu().numpy()
    assert n_copies.item() > 10
    for b, n in enumerate(-(-lens // page)):
        assert (new[b, :n] < n_live.item()).all() and np.array_equal(new[b, n:], table[b, n:])
        for c, old in zip(caches, before):
            assert np.array_equal(words(c)[new[b, :n]], old[table[b, :n]])
    # once more: nothing is left to do
    rd.rudder_page_compact(rd.PageCompactArgs(T, i32(lens), page, T, remap, copies, n_copies, n_live), handle)
    assert n_copies.item() == 0 and np.array_equal(T.cpu().numpy(), new)
    status_clean(rd)


def test_pool_bad_data_is_recorded(rd):
    table, lens = np.array([[0, 9, 2], [3, -1, 5], [1, 1, 1]], np.int32), np.array([40, 48, 49], np.int32)      # page 9 of 9, -1, one page too long
    want = shared.release(table, lens, 16, [], 9)
    refs, free, n_free = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (9, 9, 1))
    for L, code in ((lens, None), (np.array([8, 8, 49], np.int32), rd.BAD_LENGTH), (np.array([8, -3, 8], np.int32), rd.BAD_LENGTH), (np.array([40, 8, 8], np.int32), rd.BAD_PAGE)):
        rd.rudder_page_release(rd.PageReleaseArgs(i32(table), i32(L), 16, refs, free, n_free))
        last, where = rd.rudder_device_status()
        assert last == rd.ERR_ARG and (code is None or where == code)
        want = shared.release(table, np.minimum(L, 48), 16, [], 9)
        assert np.array_equal(refs.cpu().numpy(), want[1]) and np.array_equal(free.cpu().numpy(), want[2])
    rd.rudder_page_release(rd.PageReleaseArgs(i32(table), i32([8, 8, 8]), 16, refs, free, n_free, drop=i32([3])))
    assert rd.rudder_device_status() == (rd.ERR_ARG, rd.BAD_LENGTH)
    new, remap, copies, n_copies, n_live = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((3, 3), (9,), (4, 3), (1,), (1,)))
    rd.rudder_page_compact(rd.PageCompactArgs(i32(table), i32([40, 48, 48]), 16, new, remap, copies, n_copies, n_live))
    assert rd.rudder_device_status() == (rd.ERR_ARG, rd.BAD_PAGE)
    assert np.array_equal(new.cpu().numpy(), shared.compact(table, np.array([40, 48, 48]), 16, 9)[0])


def test_refused_on_another_device(rd):
    cpu = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(rd.RudderError):
        rd.PageReleaseArgs(i32([[0]]), i32([1]), 16, i32([0]), i32([0]), cpu)


# ---- attention with a shared prefix -------------------------------------------------------------------------------------------

class Shared(Attention):
    """Groups [(prefix, [(tokens behind it, new tokens), ...]), ...]: requests whose first `prefix` tokens are those of a parent, whose row stands behind
    those of the requests.  Full pages are the parent's own; the rest of a page is copied.  A negative number of tokens: shorter than the prefix."""

    def __init__(self, rd, groups, heads, kv, D, page, fmt, seed=0, order="heads", dead=float("nan")):
        lens = [max(0, p + n) for p, members in groups for n, _ in members]
        q_lens = [q for _, members in groups for _, q in members]
        parents = [p for p, _ in groups]
        super().__init__(rd, lens + parents, q_lens + [0] * len(parents), heads, kv, D, page, fmt, seed=seed, order=order, dead=dead)
        self.B, self.prefix = len(lens), parents
        self.starts = np.concatenate([[0], np.cumsum([len(m) for _, m in groups])])
        for g, p in enumerate(parents):
            up = self.B + g
            for b in range(self.starts[g], self.starts[g + 1]):
                n = min(p, lens[b])
                full, rest = divmod(n, page)
                self.table[b, :full] = self.table[up, :full]
                if rest:
                    for c in (self.kc, self.vc):
                        c[int(self.table[b, full]), :, :rest] = c[int(self.table[up, full]), :, :rest]
                for store in (self.k, self.v):
                    store[b][:n] = store[up][:n]
        self.lens, self.q_lens = lens, q_lens

    def run_shared(self, causal, starts=True, pad=0, q_pad=0, group_q=None, n_groups=None, prefix=None, rows=None, stream=None):
        rd, M, width, B = self.rd, sum(self.q_lens), self.heads * self.D, self.B
        Q = torch.zeros((M + pad, width + q_pad), dtype=torch.bfloat16, device="cuda")
        Q[:M, :width] = to_dev_bf16(self.qb)
        O = torch.full((M + pad, width + 2 * q_pad), 5.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((M + pad, self.heads), 5.0, device="cuda")
        s = i32(np.concatenate([[0], np.cumsum(self.q_lens)])) if starts else None
        table = i32(self.table)
        attn = rd.AttentionArgs(Q[:, :width], self.heads, self.cache, table[:B], i32(self.lens), self.scale, O[:, :width], q_starts=s, max_q=max(1, max(self.q_lens)),
                                causal=causal, lse=lse)
        G = len(self.prefix) if n_groups is None else n_groups
        most = max(sum(self.q_lens[self.starts[g]:self.starts[g + 1]]) for g in range(len(self.prefix)))
        self.args = rd.SharedAttentionArgs(attn, i32(self.starts[:G + 1]), i32((self.prefix if prefix is None else prefix)[:G]),
                                           i32(([B + g for g in range(G)] if rows is None else rows)[:G]), max(1, most) if group_q is None else group_q, page_table=table)
        rd.rudder_attention_shared(self.args, stream=stream)
        torch.cuda.synchronize()
        assert (O[M:] == 5.0).all().item() and (O[:, width:] == 5.0).all().item() and (lse[M:] == 5.0).all().item()
        self.O, self.lse = O, lse
        return glue.bf16_to_f32(bf16_to_np(O[:M, :width])).astype(np.float64).reshape(M, self.heads, self.D), lse[:M].cpu().numpy().astype(np.float64)


    def check_far_apart(self, o, lse, causal):
        """check() for scores far apart.  An E4M3 cache's probabilities are f16 numbers: below 2^-25 of the row's largest (which is at most 1) they are off by up to
        2^-36 of it each, so a channel in which every larger one meets a value of zero may be off by (number of keys) 2^-36 max |v|."""
        q = glue.bf16_to_f32(self.qb).astype(np.float64).reshape(-1, self.heads, self.D)
        ep, at = (2.0 ** -15 if self.fmt == "bf16" else 2.0 ** -10), 0
        for b, n in enumerate(self.q_lens):
            wo, wl_, a, ds = paged.attention(q[at:at + n], self.k[b], self.v[b], self.scale, causal)
            es = ds * (self.D + 4) * 2 * U
            floor = 0.0 if self.fmt == "bf16" or not self.lens[b] else self.lens[b] * 2.0 ** -36 * np.abs(self.v[b]).max()
            assert (np.abs(o[at:at + n] - wo) <= 2.0 ** -8 * np.abs(wo) + a * (2 * es[..., None] + ep + 2.0 ** -18) + floor + 1e-38).all(), b
            assert (np.abs(lse[at:at + n] - wl_) <= es + 2.0 ** -20 * (1 + np.abs(wl_)) + self.lens[b] * U).all(), b
            at += n


def same(n, own, q):
    return [(own, q)] * n


GROUPS = [
    [(320, same(8, 7, 1))],                                                                        # eight candidates
    [(0, same(2, 5, 1)), (1, [(0, 1), (1, 1)]), (16, []), (47, [(3, 1), (0, 1), (200, 1)])],        # no prefix, a prefix of one, an empty group, nothing behind it
    [(1000, [(1, 1), (-400, 1), (-1000, 1), (30, 1)]), (129, same(5, 40, 1))],                      # requests shorter than the prefix, one of them empty
    [(700, [(9, 3), (3, 3), (2, 3), (80, 1), (5, 0)]), (64, [(20, 5), (6, 4), (1, 2)])],            # ragged new tokens, more of them than the request has of its own
]


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads,kv,D,page", [(4, 4, 128, 16), (8, 2, 64, 32), (3, 1, 256, 8), (16, 1, 128, 64), (8, 8, 64, 1)])
@pytest.mark.parametrize("groups", range(len(GROUPS)))
def test_shared(rd, groups, heads, kv, D, page, causal, fmt):
    a = Shared(rd, GROUPS[groups], heads, kv, D, page, fmt, seed=groups + D)
    o, lse = a.run_shared(causal, pad=2, q_pad=8)
    a.check(o, lse, causal)
    status_clean(rd)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,kv,D,page,n,T,prefix,own", [
    (2, 2, 128, 64, 10, 16, 1500, 40), (4, 1, 64, 16, 5, 33, 300, 100), (2, 1, 256, 32, 7, 20, 777, 64), (1, 1, 128, 128, 40, 5, 5000, 3), (16, 2, 128, 16, 3, 40, 200, 500)])
@pytest.mark.parametrize("causal", [False, True])
def test_shared_many_rows(rd, heads, kv, D, page, n, T, prefix, own, causal, fmt):
    """More than 32 rows on either side of the cut, or on both: prefixes at any place of a page and of a tile."""
    rng = np.random.default_rng(T)
    groups = [(p, [(int(rng.integers(T, T + own)), int(rng.integers(1, T + 1))) for _ in range(n)]) for p in (prefix, prefix // 2 + 1)]
    a = Shared(rd, groups, heads, kv, D, page, fmt, seed=T)
    o, lse = a.run_shared(causal, pad=1)
    a.check(o, lse, causal)
    status_clean(rd)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("n_groups,each", [(31, 1), (33, 1), (3, 50), (40, 3), (300, 2)])
def test_shared_counts(rd, n_groups, each, fmt):
    """Both ways of finding a request's group, for one and for many requests."""
    rng = np.random.default_rng(n_groups)
    groups = [(int(rng.integers(0, 900)), [(int(rng.integers(1, 60)), int(rng.integers(1, 3))) for _ in range(int(rng.integers(0, each + 1)))]) for _ in range(n_groups)]
    groups[0] = (500, same(each, 9, 2))
    a = Shared(rd, groups, 4, 2, 64, 16, fmt, seed=each)
    o, lse = a.run_shared(True)
    a.check(o, lse, True)
    o2, lse2 = a.run_shared(True)
    assert np.array_equal(o, o2) and np.array_equal(lse, lse2)     # nothing depends on timing
    status_clean(rd)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_shared_and_paged_agree(rd, fmt):
    """The same arguments to both, with and without a prefix.  (Not bit for bit: the keys are added up in another order, and 32-bit sums depend on it.  Both
    stay within the bounds of the definition.)"""
    a = Shared(rd, [(300, [(20, 1), (5, 1)]), (64, [(8, 1)])], 4, 2, 128, 16, fmt)
    for prefix in ([0, 0], None):
        o, lse = a.run_shared(False, prefix=prefix)
        a.check(o, lse, False)
    a.O.fill_(7.0)
    rd.rudder_attention_paged(a.args.attn)
    a.check(glue.bf16_to_f32(bf16_to_np(a.O)).astype(np.float64).reshape(o.shape), a.lse.cpu().numpy().astype(np.float64), False)
    status_clean(rd)


def test_shared_hints_and_groups_that_cover_not_all(rd):
    a = Shared(rd, [(400, same(6, 9, 3)), (90, same(9, 30, 2))], 8, 2, 128, 16, "bf16")
    for kw in (dict(group_q=1), dict(group_q=3), dict(group_q=1000), dict(n_groups=1), dict(starts=True)):
        o, lse = a.run_shared(True, **kw)
        a.check(o, lse, True)
    status_clean(rd)


def test_shared_without_q_starts_and_over_queries(rd):
    a = Shared(rd, [(333, same(4, 9, 2)), (64, same(3, 30, 2))], 4, 4, 64, 16, "bf16")
    o, lse = a.run_shared(True)
    o2, lse2 = a.run_shared(True, starts=False)
    assert np.array_equal(o, o2) and np.array_equal(lse, lse2)
    attn = a.args.attn
    Q = attn.keep[0]
    X = Q.contiguous().clone()
    over = rd.AttentionArgs(X, 4, a.cache, attn.keep[1], attn.keep[2], a.scale, X, max_q=2, causal=True)
    rd.rudder_attention_shared(rd.SharedAttentionArgs(over, *a.args.keep[:3], 8, page_table=a.args.keep[3]))
    assert np.array_equal(glue.bf16_to_f32(bf16_to_np(X)).reshape(o.shape), o)
    status_clean(rd)


def test_shared_bad_groups_are_recorded(rd):
    a = Shared(rd, [(333, same(4, 9, 2)), (64, same(3, 30, 2))], 4, 2, 64, 16, "bf16", dead=0.0)
    width = a.table.shape[1] * 16
    for kw, exact in ((dict(prefix=[333, -5]), True), (dict(prefix=[333, width + 1]), True), (dict(rows=[a.B, a.B + 2]), True), (dict(rows=[-1, a.B + 1]), True)):
        o, lse = a.run_shared(True, **kw)
        assert rd.rudder_device_status() == (rd.ERR_ARG, rd.BAD_LENGTH)
        a.check(o, lse, True)                                      # such a group shares nothing
    keep = a.starts
    for starts in ([-2, 4, 7], [0, 4, 99], [3, 1, 7], [0, 9, 5]):
        a.starts = np.array(starts)
        try:
            o, _ = a.run_shared(True, group_q=8)
        finally:
            a.starts = keep
        assert rd.rudder_device_status()[0] in (rd.OK, rd.ERR_ARG) and o.shape[0] == 14
    o, lse = a.run_shared(True)
    a.check(o, lse, True)
    status_clean(rd)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,kv,T", [(4, 2, 2), (4, 1, 12)])
def test_shared_captured_follows_the_lengths(rd, heads, kv, T, fmt):
    """A captured call replayed with other prefixes and lengths: the device's data decide.  Two graphs share the workspace."""
    a = Shared(rd, [(700, same(5, 40, T)), (333, same(4, 30, T))], heads, kv, 128, 16, fmt)
    o1, l1 = a.run_shared(True)
    args, O = a.args, a.O
    ws = torch.empty(rd.rudder_attention_shared_workspace_bytes(args) + 256, dtype=torch.uint8, device="cuda")
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g):
            rd.rudder_attention_shared(args, ws)
    want = O.clone()
    prefix, lens = args.keep[1], args.attn.keep[2]
    for p, cut in (([700, 333], 0), ([512, 0], 0), ([0, 0], 0), ([650, 333], 8), ([700, 333], 0)):
        prefix.copy_(i32(p))
        lens.copy_(i32([n - cut for n in a.lens]))
        for g in graphs:
            ws.fill_(255)
            O.fill_(3.0)
            g.replay()
            got = glue.bf16_to_f32(bf16_to_np(O)).astype(np.float64).reshape(o1.shape)
            if cut == 0:
                a.check(got, l1, True)
            if p == [700, 333]:
                assert torch.equal(O, want)
    status_clean(rd)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("scale", [3.0, -3.0, 0.0, -0.05])
@pytest.mark.parametrize("heads,kv,D,n,T,prefix", [(2, 2, 128, 20, 16, 900), (4, 1, 64, 9, 20, 700), (4, 2, 128, 9, 1, 900), (2, 1, 256, 7, 20, 300), (16, 1, 64, 6, 1, 500), (2, 2, 128, 3, 40, 400)])
def test_shared_scales_of_any_sign(rd, heads, kv, D, n, T, prefix, scale, fmt):
    """Large scores, whose running maximum is raised again and again, and factors below and at zero, on every kernel of either pass."""
    rng = np.random.default_rng(n)
    a = Shared(rd, [(prefix, [(int(rng.integers(T, T + 90)), T) for _ in range(n)]), (prefix // 3, same(2, T + 3, T))], heads, kv, D, 16, fmt, seed=n)
    a.scale = scale
    o, lse = a.run_shared(True)
    a.check_far_apart(o, lse, True)
    status_clean(rd)


@pytest.mark.parametrize("T", [1, 40])
def test_shared_far_pages(rd, T):
    """Pages behind 2^31 elements and 2^32 bytes: attention, and a copy between them."""
    page, kv, D = 64, 8, 128
    n_pages = int(2.8e9) // (page * kv * D) + 1
    a = Attention(rd, [333, 320, 330], [T, T, T], 8, kv, D, page, "bf16", seed=4, far=n_pages)
    for b in (1, 2):
        a.table[b, :3] = a.table[0, :3]
        for store in (a.k, a.v):
            store[b][:192] = store[0][:192]
    a.run(True)
    attn = a.args
    a.O.fill_(7.0)
    rd.rudder_attention_shared(rd.SharedAttentionArgs(attn, i32([0, 3]), i32([192]), i32([2]), 3 * T))
    a.check(glue.bf16_to_f32(bf16_to_np(a.O)).astype(np.float64).reshape(3 * T, 8, D), a.lse.cpu().numpy().astype(np.float64), True)
    src, dst = n_pages - 1, n_pages - 9
    a.vc[src] = torch.randn((kv, page, D), device="cuda").to(torch.bfloat16)
    a.vc[dst] = 1.0
    rd.rudder_page_copy(rd.PageCopyArgs(i32([[src, dst, 50]])), rd.PagedCaches([a.cache]))
    assert torch.equal(a.vc[dst, :, :50], a.vc[src, :, :50]) and (a.vc[dst, :, 50:] == 1.0).all().item()
    status_clean(rd)


# ---- low-rank adapters ------------------------------------------------------------------------------------------------------

class Lora:
    def __init__(self, rd, M, K, N, R, n, adapters, ranks, seed=0, pads=(0, 0, 0), base="other"):
        rng = np.random.default_rng(seed)
        bf = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(torch.bfloat16)  # noqa: E731
        self.rd, self.adapters, self.ranks = rd, np.asarray(adapters, np.int32), np.asarray(ranks, np.int32)
        X, A, B, base_ = bf(M, K + pads[0]), bf(n, R, K + pads[1]), bf(n, N, R), bf(M, N + pads[2])
        for a in range(n):                                         # what stands behind an adapter's rank is not its own
            A[a, min(max(ranks[a], 0), R):] = float("nan")
            B[a, :, min(max(ranks[a], 0), R):] = float("inf")
        self.scales = rng.standard_normal(n).astype(np.float32)
        self.dev = [t.cuda() for t in (X, A, B, base_)]
        self.host = [t.float().numpy() for t in (X[:, :K], A[:, :, :K], B, base_[:, :N])]
        self.X, self.A, self.B = self.dev[0][:, :K], self.dev[1][:, :, :K], self.dev[2]
        self.K, self.R, self.N, self.M = K, R, N, M
        self.buf = torch.full((M, N + pads[2]), 7.0, dtype=torch.bfloat16, device="cuda")
        if base == "same":
            self.buf.copy_(self.dev[3])
        self.Y = self.buf[:, :N]
        self.base = {"none": None, "same": self.Y, "other": self.dev[3][:, :N]}[base]
        if base == "none":
            self.host[3] = np.zeros_like(self.host[3])
        self.args = rd.LoraArgs(self.X, self.A, self.B, i32(self.ranks), cuda(self.scales), i32(self.adapters), self.base, self.Y)

    def run(self, workspace=None, stream=None):
        self.rd.rudder_lora(self.args, workspace, stream)
        torch.cuda.synchronize()
        return glue.bf16_to_f32(bf16_to_np(self.Y.contiguous())).astype(np.float64)

    def check(self, y, base=None):
        ranks = np.clip(self.ranks, 0, self.R)
        want, s = shared.lora(self.host[0], self.host[1], self.host[2], ranks, self.scales, self.adapters, self.host[3] if base is None else base)
        assert np.isfinite(y).all()
        bound = 2.0 ** -8 * np.abs(want) + s * (2.0 ** -16 + (self.K + 2 * self.R + 16) * 2 * U)
        assert (np.abs(y - want) <= bound + 1e-38).all(), (np.abs(y - want) / bound).max()


def rows_of(rng, M, n, run):
    rows = []
    while len(rows) < M:
        rows += [int(rng.integers(-1, n))] * run
    return rows[:M]


@pytest.mark.parametrize("M,K,N,R,n,run", [
    (1, 64, 64, 8, 1, 1), (1, 2048, 6144, 16, 8, 1), (3, 8, 8, 8, 2, 1), (7, 136, 72, 16, 3, 1), (16, 512, 264, 24, 5, 2), (17, 1000, 120, 64, 4, 1), (33, 256, 1000, 40, 9, 3),
    (64, 2048, 512, 128, 20, 1), (64, 384, 128, 256, 2, 64), (65, 256, 136, 16, 3, 1), (200, 520, 264, 64, 40, 1), (500, 1024, 520, 72, 7, 77), (1111, 128, 256, 128, 1, 1),
    (300, 4096, 64, 256, 3, 100), (2000, 64, 128, 8, 4096, 1), (129, 2000, 1032, 32, 2, 64)])
def test_lora(rd, M, K, N, R, n, run):
    rng = np.random.default_rng(M + K)
    ranks = rng.integers(0, R + 1, n)
    ranks[0] = R
    a = Lora(rd, M, K, N, R, n, rows_of(rng, M, n, run), ranks, seed=M)
    y = a.run()
    a.check(y)
    assert np.array_equal(y, a.run())                              # (base is another buffer)
    status_clean(rd)


@pytest.mark.parametrize("M", [1, 5, 64, 100])
@pytest.mark.parametrize("base", ["none", "same", "other"])
def test_lora_strides_and_bases(rd, M, base):
    rng = np.random.default_rng(M)
    a = Lora(rd, M, 264, 200, 24, 3, rows_of(rng, M, 3, 2), [24, 5, 17], seed=M, pads=(8, 24, 16), base=base)
    tail = a.buf[:, 200:].clone()
    a.check(a.run())
    assert torch.equal(a.buf[:, 200:], tail)
    status_clean(rd)


@pytest.mark.parametrize("M", [9, 90])
def test_lora_rows_do_not_meet(rd, M):
    """A row's result does not depend on what stands in the others, nor on their adapters; one without an adapter is its base bit for bit."""
    rng = np.random.default_rng(M)
    rows = np.array(rows_of(rng, M, 4, 1))
    rows[3] = 2
    rows[4] = -1
    a = Lora(rd, M, 256, 128, 16, 4, rows, [16, 9, 16, 1])
    y = a.run()
    a.check(y)
    assert np.array_equal(y[rows < 0], a.host[3][rows < 0])
    others = np.flatnonzero(np.arange(M) != 3)
    a.dev[0][torch.from_numpy(others).cuda()] = float("nan")
    a.dev[1][[0, 1, 3]] = float("inf")
    assert np.array_equal(a.run()[3], y[3])
    # the same row alone
    b = rd.LoraArgs(a.X[3:4], a.A, a.B, *a.args.keep[3:5], i32([2]), a.base[3:4], a.Y[:1])
    rd.rudder_lora(b)
    alone = glue.bf16_to_f32(bf16_to_np(a.Y[:1].contiguous()))[0]
    if M <= 64:
        assert np.array_equal(alone, y[3])
    status_clean(rd)


@pytest.mark.parametrize("M", [5, 80])
def test_lora_bad_data_is_recorded(rd, M):
    rows = np.zeros(M, np.int32)
    rows[1], rows[2], rows[3] = 4, -2, 1
    a = Lora(rd, M, 64, 64, 8, 4, rows, [8, 0, 3, 8])
    y = a.run()
    assert rd.rudder_device_status() == (rd.ERR_ARG, rd.BAD_ADAPTER)
    a.adapters = np.where((rows >= 0) & (rows < 4), rows, -1)
    a.check(y)
    for r in (9, -1):
        b = Lora(rd, M, 64, 64, 8, 2, np.zeros(M, np.int32), [r, 8])
        y = b.run()
        assert rd.rudder_device_status() == (rd.ERR_ARG, rd.BAD_ADAPTER)
        b.check(y)


@pytest.mark.parametrize("M", [4, 150])
def test_lora_infinite_inner_sum(rd, M):
    """An infinite inner sum gives the infinities of the definition, not a number that is none."""
    a = Lora(rd, M, 64, 64, 8, 1, np.zeros(M, np.int32), [1])
    a.dev[0][0, 0] = float("inf")
    a.dev[1][0, 0, 0] = 1.0
    y = a.run()
    s = np.sign(a.scales[0] * a.host[2][0, :, 0])
    assert np.array_equal(y[0], np.where(s > 0, np.inf, -np.inf)) and np.isfinite(y[1:]).all()


@pytest.mark.parametrize("M", [4, 150])
def test_lora_captured_follows_the_rows(rd, M):
    """Replays with other adapters, ranks and weights; two graphs share the workspace."""
    rng = np.random.default_rng(M)
    a = Lora(rd, M, 512, 256, 32, 6, rows_of(rng, M, 6, 1), [32, 7, 16, 0, 32, 1])
    for i in range(6):
        a.dev[1][i], a.dev[2][i] = torch.randn_like(a.dev[1][i]), torch.randn_like(a.dev[2][i])
    a.host[1], a.host[2] = a.A.float().cpu().numpy(), a.B.float().cpu().numpy()
    ws = torch.empty(rd.rudder_lora_workspace_bytes(a.args) + 256, dtype=torch.uint8, device="cuda")
    a.check(a.run(ws))
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g):
            rd.rudder_lora(a.args, ws)
    for turn in range(3):
        a.adapters = np.array(rows_of(rng, M, 6, turn + 1), np.int32)
        a.ranks = rng.integers(0, 33, 6).astype(np.int32)
        a.args.keep[5].copy_(i32(a.adapters))
        a.args.keep[3].copy_(i32(a.ranks))
        for g in graphs:
            ws.fill_(255)
            a.buf.fill_(9.0)
            g.replay()
            torch.cuda.synchronize()
            a.check(glue.bf16_to_f32(bf16_to_np(a.Y.contiguous())).astype(np.float64))
    status_clean(rd)
