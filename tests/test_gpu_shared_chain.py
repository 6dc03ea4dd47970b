"""The operators for many requests that continue one context, run together as they would be used: a context is cached, candidates fork off it, a block's rows of all
of them go through the cache with adapters beside the output projection, some end, the pool is closed up, and the next step reads the same."""
import numpy as np
import pytest
import torch

from helpers import bf16_to_np
from oracle import glue
from test_gpu_paged import rd, status_clean  # noqa: F401  (rd: the fixture)

pytestmark = pytest.mark.gpu


def i32(v):
    return torch.tensor(np.asarray(v, np.int32), device="cuda")


def as64(t):
    return glue.bf16_to_f32(bf16_to_np(t.contiguous())).astype(np.float64)


class Server:
    """Two layers' caches behind one table: row 0 the context, rows 1 .. n its candidates."""

    def __init__(self, rd, fmt, n=5, context=333, page=16, heads=8, kv=2, D=64, n_pages=120):
        self.rd, self.n, self.page, self.heads, self.kv, self.D, self.n_pages = rd, n, page, heads, kv, D, n_pages
        kind = torch.bfloat16 if fmt == "bf16" else torch.float8_e4m3fn
        g = torch.Generator(device="cuda").manual_seed(1)
        self.gen = g
        rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        self.caches = [rd.PagedCache(*(torch.full((n_pages, kv, page, D), float("nan"), device="cuda").to(kind) for _ in range(2))) for _ in range(2)]
        self.layers = rd.PagedCaches(self.caches)
        self.table = torch.full((n + 1, 40), -1, dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
        self.refs, self.free, self.n_free = (torch.zeros(k, dtype=torch.int32, device="cuda") for k in (n_pages, n_pages, 1))
        self.release = rd.PageReleaseArgs(self.table, self.lens, page, self.refs, self.free, self.n_free)
        rd.rudder_page_release(self.release)                       # nothing is held: the first free list
        angle = torch.arange(1024, device="cuda")[:, None] * 10000.0 ** (-torch.arange(0, D, 2, device="cuda") / D)
        self.cos, self.sin = torch.cos(angle).contiguous(), torch.sin(angle).contiguous()
        self.rand = rand
        self.append([0] if context else [], [context])

    def append(self, rows, new):
        """New tokens of the given requests into both layers -> (their queries of the first layer, starts)."""
        rd, counts = self.rd, np.zeros(self.n + 1, np.int32)
        counts[rows] = new
        M = int(counts.sum())
        slots, pos = torch.empty(M, dtype=torch.int64, device="cuda"), torch.empty(M, dtype=torch.int32, device="cuda")
        starts, used = torch.empty(self.n + 2, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
        rd.rudder_page_tables(rd.PageTableArgs(self.lens, i32(counts), self.free, self.table, self.page, slots, pos, starts, used))
        queries = []
        for cache in self.caches:
            X = self.rand(M, (self.heads + 2 * self.kv) * self.D).to(torch.bfloat16)
            Q = torch.empty((M, self.heads * self.D), dtype=torch.bfloat16, device="cuda")
            rd.rudder_qk_norm_rope(rd.QkArgs(X, self.heads, self.kv, self.D, None, None, 1e-6, self.cos, self.sin, rd.ROPE_HALF, pos, Q, cache=cache, slots=slots))
            queries.append(Q)
        self.lens += i32(counts)
        rd.rudder_page_release(self.release)                       # the pages taken are gone from the list
        return queries, starts

    def attend(self, Q, starts, prefix, shared):
        """Rows 0 .. n as one group behind `prefix`, or each for itself."""
        rd = self.rd
        O = torch.zeros_like(Q)
        lse = torch.zeros((Q.shape[0], self.heads), device="cuda")
        a = rd.AttentionArgs(Q, self.heads, self.caches[0], self.table, self.lens, 0.125, O, q_starts=starts, max_q=8, causal=True, lse=lse)
        if shared:
            rd.rudder_attention_shared(rd.SharedAttentionArgs(a, i32([0, self.n + 1]), i32([prefix]), i32([0]), Q.shape[0]))
        else:
            rd.rudder_attention_paged(a)
        return O, lse


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_candidates_of_one_context(rd, fmt):
    s = Server(rd, fmt)
    prefix = 333 // s.page * s.page
    free_before = s.n_free.item()
    # five candidates fork off the context: only the started page is copied
    used = torch.zeros(1, dtype=torch.int32, device="cuda")
    rd.rudder_page_fork(rd.PageForkArgs(s.table, s.lens, s.page, i32([0] * 5), i32([1, 2, 3, 4, 5]), s.free, used), s.layers)
    rd.rudder_page_release(s.release)
    assert used.item() == 5 and s.lens.tolist() == [333] * 6 and s.n_free.item() == free_before - 5
    assert sorted(set(s.refs.tolist())) == [0, 1, 6]
    # a step of new tokens for the candidates; the shared pages are not written
    (Q, _), starts = s.append([1, 2, 3, 4, 5], [3, 8, 1, 5, 7])
    O, lse = s.attend(Q, starts, prefix, True)
    want, want_lse = s.attend(Q, starts, prefix, False)
    # both within 2^-8 of the definition's value and sums' rounding of it: within 2^-7 of one another, and 2^-9 (E4M3: its probabilities') of the weighted mean of |v|
    assert (np.abs(as64(O) - as64(want)) <= 2.0 ** -7 * np.abs(as64(want)) + 2.0 ** -8).all()
    assert (lse - want_lse).abs().max().item() < 2.0 ** -12
    # adapters of two robots beside the output projection, in place
    W = torch.randn((512, 256), device="cuda") * 0.05
    w = rd.rudder_pack_weights(W, None, rd.W4A8_INT, 64)
    M = Q.shape[0]
    tab = rd.ScaleTable(torch.ones((1, 1), device="cuda"))
    Y = rd.rudder_linear(w, O[:, :256], rd.Segments([0, M], [0]), 0, tab)
    base = as64(Y)
    A, B = (torch.randn(sh, device="cuda").to(torch.bfloat16) * 0.1 for sh in ((2, 16, 256), (2, 512, 16)))
    rows = np.array([0] * 3 + [1] * 8 + [-1] * 1 + [0] * 5 + [1] * 7, np.int32)
    rd.rudder_lora(rd.LoraArgs(O[:, :256], A, B, i32([16, 9]), torch.tensor([1.0, 0.5], device="cuda"), i32(rows), Y, Y))
    x = as64(O[:, :256])
    for m, a in enumerate(rows):
        r = (16, 9)[a]
        add = 0.0 if a < 0 else (1.0, 0.5)[a] * (as64(B[a])[:, :r] @ (as64(A[a])[:r] @ x[m]))
        assert (np.abs(as64(Y[m:m + 1])[0] - (base[m] + add)) <= 2.0 ** -8 * np.abs(base[m] + add) + 1e-3).all()
    # two candidates end; the pool is closed up; the others read what they read before
    drop = rd.PageReleaseArgs(s.table, s.lens, s.page, s.refs, s.free, s.n_free, drop=i32([2, 4]))
    rd.rudder_page_release(drop)
    new = [torch.zeros(k, dtype=torch.int32, device="cuda") for k in ((s.n_pages,), (s.n_pages // 2, 3), (1,), (1,))]
    rd.rudder_page_compact(rd.PageCompactArgs(s.table, s.lens, s.page, s.table, *new), s.layers)
    n_live = new[3].item()
    assert n_live == s.n_pages - s.n_free.item()
    rd.rudder_page_release(s.release)
    assert s.free[:s.n_free.item()].tolist() == list(range(n_live, s.n_pages))
    again, again_lse = s.attend(Q, starts, prefix, True)
    keep = np.concatenate([np.arange(3), np.arange(11, 12), np.arange(17, 24)])           # rows of requests 1, 3 and 5
    assert torch.equal(again[keep], O[keep]) and torch.equal(again_lse[keep], lse[keep])
    status_clean(rd)


def test_two_streams_at_once(rd):
    """Calls on two streams with workspaces of their own, and pages of two pools."""
    ss = [Server(rd, "bf16", context=c) for c in (333, 200)]
    streams = [torch.cuda.Stream() for _ in ss]
    plans = []
    for s in ss:
        used = torch.zeros(1, dtype=torch.int32, device="cuda")
        rd.rudder_page_fork(rd.PageForkArgs(s.table, s.lens, s.page, i32([0] * 5), i32([1, 2, 3, 4, 5]), s.free, used), s.layers)
        rd.rudder_page_release(s.release)
        (Q, _), starts = s.append([1, 2, 3, 4, 5], [3, 8, 1, 5, 7])
        O = torch.zeros_like(Q)
        a = rd.AttentionArgs(Q, s.heads, s.caches[0], s.table, s.lens, 0.125, O, q_starts=starts, max_q=8, causal=True)
        sh = rd.SharedAttentionArgs(a, i32([0, s.n + 1]), i32([192]), i32([0]), Q.shape[0])
        plans.append((sh, O, torch.empty(rd.rudder_attention_shared_workspace_bytes(sh) + 256, dtype=torch.uint8, device="cuda")))
    want = []
    for sh, O, ws in plans:
        rd.rudder_attention_shared(sh, ws)
        want.append(O.clone())
    torch.cuda.synchronize()
    for _ in range(20):
        for (sh, O, ws), st in zip(plans, streams):
            rd.rudder_attention_shared(sh, ws, stream=st)
    torch.cuda.synchronize()
    for (_, O, _), w in zip(plans, want):
        assert torch.equal(O, w)
    status_clean(rd)
