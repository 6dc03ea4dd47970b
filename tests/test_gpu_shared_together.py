"""The operators for many requests that continue one context, on the GPU: calls on two streams at once that each have to write all of their outputs, replays with shorter
requests, and groups that are partly sound."""
import numpy as np
import pytest
import torch

from helpers import bf16_to_np
from oracle import glue, shared
from test_gpu_paged import rd, status_clean  # noqa: F401  (rd: the fixture)
from test_gpu_shared import Lora, Shared, i32, layers, pool, rows_of, same, words

pytestmark = pytest.mark.gpu


def f64(t):
    return glue.bf16_to_f32(bf16_to_np(t.contiguous())).astype(np.float64)


class Work:
    """One user's buffers: attention over its groups, adapters, a fork and a compaction of its pool; each call's outputs are overwritten in front of it, on its stream."""

    def __init__(self, rd, seed, fmt):
        rng = np.random.default_rng(seed)
        self.rd = rd
        self.a = Shared(rd, [(700 + 33 * seed, same(9, 40, 3)), (64, same(5, 3000, 3))], 8, 2, 128, 16, fmt, seed=seed)
        o, lse = self.a.run_shared(True)
        self.a.check(o, lse, True)
        self.attn, self.O, self.lse = self.a.args, self.a.O, self.a.lse
        self.loras = [Lora(rd, M, 512, 2056, 40, 5, rows_of(rng, M, 5, 2), [40, 0, 9, 33, 1], seed=seed + M) for M in (20 + seed, 400 + seed)]
        for l in self.loras:
            l.check(l.run())
        table, lens, n_pages = pool(rng, 6, 16, 400, share=0.5, spare=60)
        lens[0] = max(lens[0], 17) if table[0, 1] >= 0 else lens[0]
        free = np.setdiff1d(np.arange(n_pages), table).astype(np.int32)
        self.T0 = np.concatenate([table, np.full((20, table.shape[1]), -5, np.int32)])
        self.L0 = np.concatenate([lens, np.zeros(20, np.int32)])
        src, dst = rng.integers(0, 6, 20).astype(np.int32), (6 + np.arange(20)).astype(np.int32)
        self.caches, handle = layers(rd, 3, n_pages, 4, 16, 64, fmt, seed=seed)
        self.handle, self.before = handle, [c.clone() for c in self.caches]
        host = [words(c) for c in self.before]
        self.T, self.L, self.used = i32(self.T0), i32(self.L0), i32([0])
        self.fork = rd.PageForkArgs(self.T, self.L, 16, i32(src), i32(dst), i32(free), self.used)
        t1, l1, copies, n = shared.fork(self.T0, self.L0, 16, src.tolist(), dst.tolist(), free, None, 0)
        host = [shared.copy_tokens(h, copies) for h in host]
        t2, remap, moves, live = shared.compact(t1, l1, 16, n_pages)
        self.N, self.remap, self.moves, self.counts = i32(t1), i32(np.zeros(n_pages)), i32(np.zeros((n_pages // 2, 3))), i32([0, 0])
        self.compact = rd.PageCompactArgs(self.T, self.L, 16, self.N, self.remap, self.moves, self.counts[:1], self.counts[1:])
        self.want_pages = (t1, l1, [n], t2, remap, [len(moves), live], [shared.copy_tokens(h, moves) for h in host])
        self.table0, self.lens0 = i32(self.T0), i32(self.L0)
        self.ws = [torch.empty(n + 256, dtype=torch.uint8, device="cuda") for n in
                   (rd.rudder_attention_shared_workspace_bytes(self.attn), *(rd.rudder_lora_workspace_bytes(l.args) for l in self.loras))]
        torch.cuda.synchronize()
        self.want = [t.clone() for t in (self.O, self.lse, *(l.buf for l in self.loras))]
        self.seen = []

    def go(self, stream):
        rd = self.rd
        with torch.cuda.stream(stream):
            for t in (self.O, self.lse, *(l.buf for l in self.loras)):
                t.fill_(-3.0)
            for t in (self.N, self.remap, self.counts, self.used):
                t.fill_(-77)
            self.T.copy_(self.table0)
            self.L.copy_(self.lens0)
            for c, b in zip(self.caches, self.before):
                c.view(torch.uint8 if c.element_size() == 1 else torch.int16).copy_(b.view(torch.uint8 if b.element_size() == 1 else torch.int16))
            for w in self.ws:
                w.fill_(255)
        rd.rudder_attention_shared(self.attn, self.ws[0], stream=stream)
        rd.rudder_page_fork(self.fork, self.handle, stream=stream)
        for l, w in zip(self.loras, self.ws[1:]):
            rd.rudder_lora(l.args, w, stream=stream)
        rd.rudder_page_compact(self.compact, self.handle, stream=stream)
        with torch.cuda.stream(stream):
            self.seen.append([t.clone() for t in (self.O, self.lse, *(l.buf for l in self.loras), self.T, self.L, self.used, self.N, self.remap, self.counts, *self.caches)])

    def check(self):
        n = len(self.want)
        t1, l1, used, t2, remap, counts, host = self.want_pages
        for seen in self.seen:
            assert all(torch.equal(a, b) for a, b in zip(seen[:n], self.want))
            for got, want in zip(seen[n:n + 6], (t1, l1, used, t2, remap, counts)):
                assert np.array_equal(got.cpu().numpy().reshape(np.shape(want)), want)
            for got, want in zip(seen[n + 6:], host):
                assert np.array_equal(words(got), want)
        self.seen = []


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_two_streams_write_all_of_their_outputs(rd, fmt):
    both = [Work(rd, seed, fmt) for seed in (1, 2)]
    streams = [torch.cuda.Stream() for _ in both]
    torch.cuda.synchronize()
    for _ in range(6):
        for w, st in zip(both, streams):
            w.go(st)
    torch.cuda.synchronize()
    for w in both:
        w.check()
    status_clean(rd)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,kv,T", [(4, 2, 2), (4, 1, 12), (8, 1, 40)])
def test_replays_with_shorter_requests(rd, heads, kv, T, fmt):
    """A captured call follows the lengths: compared with the definition at each of them."""
    a = Shared(rd, [(700, same(5, 60, T)), (333, same(4, 50, T))], heads, kv, 128, 16, fmt)
    o1, _ = a.run_shared(True)
    args, O, L = a.args, a.O, a.lse
    ws = torch.empty(rd.rudder_attention_shared_workspace_bytes(args) + 256, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rd.rudder_attention_shared(args, ws)
    prefix, lens = args.keep[1], args.attn.keep[2]
    full, k, v = list(a.lens), a.k, a.v
    for p, cut in (([650, 333], 8), ([700, 333], 45), ([700, 100], 300), ([64, 64], 333), ([700, 333], 0)):
        prefix.copy_(i32(p))
        a.lens = [n - cut for n in full]
        a.k, a.v = [x[:n - cut] for x, n in zip(k, full)], [x[:n - cut] for x, n in zip(v, full)]
        lens.copy_(i32(a.lens))
        ws.fill_(255)
        O.fill_(3.0)
        L.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        a.check(f64(O).reshape(o1.shape), L.cpu().numpy().astype(np.float64), True)
    status_clean(rd)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("T", [2, 40])
def test_sound_requests_beside_bad_groups(rd, T, fmt):
    """Groups that begin in front of the first request, end behind the last one or in front of their own beginning are recorded, and no request of another group is touched by them."""
    a = Shared(rd, [(333, same(4, 60, T)), (64, same(3, 70, T))], 4, 2, 64, 16, fmt)
    right, lse = a.run_shared(True)
    a.check(right, lse, True)
    for starts, sound in (([-2, 4, 7], range(7)), ([0, 4, 99], range(7)), ([3, 1, 7], (0, 4, 5, 6)), ([0, 9, 5], range(4))):
        a.starts = np.array(starts)
        try:
            o, l = a.run_shared(True, group_q=4 * T)
        finally:
            a.starts = np.array([0, 4, 7])
        assert rd.rudder_device_status() == (rd.ERR_ARG, rd.BAD_LENGTH), starts
        rows = np.concatenate([np.arange(b * T, (b + 1) * T) for b in sound])
        part = [a.lens, a.q_lens, a.k, a.v, a.qb]
        try:
            a.lens, a.q_lens, a.k, a.v = ([x[b] for b in sound] for x in part[:4])
            a.qb = part[4][rows]
            a.check(o[rows], l[rows], True)
        finally:
            a.lens, a.q_lens, a.k, a.v, a.qb = part
    status_clean(rd)
