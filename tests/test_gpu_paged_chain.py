"""The serving operators together, as a denoising step uses them: page tables -> QKV -> norm, rotation, append -> attention -> O,
step by step against the oracle, as rudder_block_cached against the same calls one by one, captured into graphs that share a
workspace, and on two streams at once."""
import numpy as np
import pytest
import torch

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


class Step:
    """B requests with a cache of their own, `new` tokens each, the four linears of a block and everything between."""

    def __init__(self, rd, old, new, heads=4, kv=2, D=64, page=16, fmt="bf16", scheme="w4a8", G=64, seed=0, pad=0, causal=False):
        self.rd, self.heads, self.kv, self.D, self.page, self.causal = rd, heads, kv, D, page, causal
        self.old, self.new = np.array(old), np.array(new)
        B, n_new = len(old), int(self.new.sum())
        self.M = n_new + pad
        H, F = heads * D, 512
        shapes = [(H, (heads + 2 * kv) * D), (heads * D, H), (H, F), (F, H)]
        self.layers = [GpuLinear(rd, wl.tiny(seed=seed + 40 + i, M=self.M, K=K, N=N, T=2), scheme, G if G else K) for i, (K, N) in enumerate(shapes)]
        rng = np.random.default_rng(seed)
        want = -(-(self.old + self.new) // page)
        held = -(-self.old // page)
        n_pages = int(want.sum()) + 4
        ids = rng.permutation(n_pages).astype(np.int32)
        table = np.full((B, int(want.max()) + 1), -1, np.int32)
        at = 0
        for b in range(B):
            table[b, :held[b]] = ids[at:at + held[b]]
            at += held[b]
        self.free = ids[at:]
        kind = torch.bfloat16 if fmt == "bf16" else torch.float8_e4m3fn
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.kc = torch.randn((n_pages, kv, page, D), generator=g, device="cuda").to(kind)
        self.vc = torch.randn((n_pages, kv, page, D), generator=g, device="cuda").to(kind)
        sc = (torch.full((kv,), 0.05, device="cuda"), torch.full((kv,), 0.1, device="cuda")) if fmt == "e4m3" else (None, None)
        self.cache = rd.PagedCache(self.kc, self.vc, *sc)
        dev = lambda a, t: torch.from_numpy(np.ascontiguousarray(a)).to(t).cuda()  # noqa: E731
        self.table = dev(table, torch.int32)
        self.slots = torch.empty(self.M, dtype=torch.int64, device="cuda")
        self.pos = torch.empty(self.M, dtype=torch.int32, device="cuda")
        self.starts, self.used = torch.empty(B + 1, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
        self.lens = dev(self.old + self.new, torch.int32)
        self.tables = rd.PageTableArgs(dev(self.old, torch.int32), dev(self.new, torch.int32), dev(self.free, torch.int32), self.table, page, self.slots, self.pos,
                                       self.starts, self.used)
        self.qw = 1 + 0.1 * torch.randn(D, generator=g, device="cuda")
        self.kw = 1 + 0.1 * torch.randn(D, generator=g, device="cuda")
        self.norm1 = 1 + 0.1 * torch.randn(H, generator=g, device="cuda")
        self.norm2 = 1 + 0.1 * torch.randn(H, generator=g, device="cuda")
        ang = torch.arange(4096, device="cuda", dtype=torch.float64)[:, None] * 100.0 ** (-torch.arange(D // 2, device="cuda", dtype=torch.float64) * 2 / D)
        self.cos, self.sin = torch.cos(ang).float(), torch.sin(ang).float()
        self.H, self.scale = H, D ** -0.5
        self.X = self.layers[0].X
        self.max_q = int(self.new.max())

    def fresh(self):
        """Output buffers and the arguments of the fused path."""
        rd, M = self.rd, self.M
        ys = [torch.full((M, l.w.N), float("nan"), dtype=torch.bfloat16, device="cuda") for l in self.layers]
        bargs = rd.BlockArgs([l.w for l in self.layers], [l.tab for l in self.layers], [l.bias for l in self.layers], [self.X, None, None, None], ys)
        lse = torch.full((M, self.heads), 9.0, device="cuda")
        qk = rd.QkArgs(None, self.heads, self.kv, self.D, self.qw, self.kw, 1e-6, self.cos, self.sin, rd.ROPE_HALF, self.pos, None, cache=self.cache, slots=self.slots)
        at = rd.AttentionArgs(None, self.heads, self.cache, self.table, self.lens, self.scale, None, q_starts=self.starts, max_q=self.max_q, causal=self.causal, lse=lse)
        ws = torch.empty(rd.rudder_block_cached_workspace_bytes(bargs, at, M) + 256, dtype=torch.uint8, device="cuda")
        return ys, bargs, lse, qk, at, ws, torch.full((M, self.H), float("nan"), dtype=torch.bfloat16, device="cuda")

    def one_by_one(self, step):
        """The same step with the public calls, one after another."""
        rd, M, L = self.rd, self.M, self.layers
        seg = L[0].seg
        n1 = rd.rudder_rmsnorm(self.X, self.norm1, 1e-6)
        y0 = rd.rudder_linear(L[0].w, n1, seg, step, L[0].tab, L[0].bias)
        q = torch.zeros((M, self.heads * self.D), dtype=torch.bfloat16, device="cuda")
        o = torch.zeros_like(q)
        lse = torch.full((M, self.heads), 9.0, device="cuda")
        rd.rudder_qk_norm_rope(rd.QkArgs(y0, self.heads, self.kv, self.D, self.qw, self.kw, 1e-6, self.cos, self.sin, rd.ROPE_HALF, self.pos, q, cache=self.cache, slots=self.slots))
        rd.rudder_attention_paged(rd.AttentionArgs(q, self.heads, self.cache, self.table, self.lens, self.scale, o, q_starts=self.starts, max_q=self.max_q, causal=self.causal, lse=lse))
        y1 = rd.rudder_linear(L[1].w, o, seg, step, L[1].tab, L[1].bias)
        h = rd.rudder_add(self.X, y1)
        y2 = rd.rudder_linear(L[2].w, rd.rudder_rmsnorm(h, self.norm2, 1e-6), seg, step, L[2].tab, L[2].bias)
        y3 = rd.rudder_linear(L[3].w, rd.rudder_gelu(y2), seg, step, L[3].tab, L[3].bias)
        return [y0, y1, y2, y3], q, o, lse, rd.rudder_add(h, y3)

    def fused(self, state, step, stream=None):
        ys, bargs, lse, qk, at, ws, out = state
        self.rd.rudder_page_tables(self.tables, stream=stream)
        self.rd.rudder_block_cached(bargs, self.norm1, self.norm2, 1e-6, out, qk, at, self.M, self.layers[0].seg, step, ws, stream=stream)


CASES = [dict(old=[40, 0, 7, 130], new=[5, 3, 0, 9]), dict(old=[700], new=[16], causal=True, heads=4, kv=4, D=128, fmt="e4m3"),
         dict(old=[31, 64], new=[1, 1], scheme="nvfp4", G=16, pad=2), dict(old=[3, 90, 12], new=[30, 1, 40], heads=8, kv=1, causal=True, scheme="w4a4", G=0)]


@pytest.mark.parametrize("kw", CASES)
def test_block_cached(rd, kw):
    s = Step(rd, **kw)
    rd.rudder_page_tables(s.tables)
    k0, v0 = s.kc.clone(), s.vc.clone()
    ys, q, o, lse, out = s.one_by_one(1)
    k1, v1 = s.kc.clone(), s.vc.clone()
    s.kc.copy_(k0), s.vc.copy_(v0)
    state = s.fresh()
    s.fused(state, 1)
    torch.cuda.synchronize()
    assert torch.equal(s.kc.view(torch.uint8), k1.view(torch.uint8)) and torch.equal(s.vc.view(torch.uint8), v1.view(torch.uint8))
    for a, b in zip(state[0], ys):
        assert torch.equal(a, b)
    assert torch.equal(state[2], lse) and torch.equal(state[6], out)
    last, where = rd.rudder_device_status()
    assert last == 0, (last, where)
    # and against the oracle, from the QKV output on
    old, new = s.old, s.new
    heads, kv, D = s.heads, s.kv, s.D
    pos, slots = s.pos.cpu().numpy(), s.slots.cpu().numpy()
    qn, kn, vn = paged.qk_norm_rope(glue.bf16_to_f32(bf16_to_np(ys[0])), heads, kv, D, s.qw.cpu().numpy(), s.kw.cpu().numpy(), 1e-6, s.cos.cpu().numpy(), s.sin.cpu().numpy(), D,
                                    False, pos)
    real = pos >= 0
    assert real.sum() == new.sum()
    assert np.array_equal(bf16_to_np(q)[real], glue.f32_to_bf16(qn.reshape(s.M, -1))[real])
    ks, vs = (0.05, 0.1) if s.kc.dtype != torch.bfloat16 else (1.0, 1.0)
    kc, vc = k1.float().cpu().numpy().astype(np.float64) * np.float32(ks), v1.float().cpu().numpy().astype(np.float64) * np.float32(vs)
    table = s.table.cpu().numpy()
    at = 0
    for b in range(len(old)):
        n, T = int(old[b] + new[b]), int(new[b])
        ids = table[b, :-(-n // s.page)]
        K = kc[ids].transpose(0, 2, 1, 3).reshape(-1, kv, D)[:n]
        V = vc[ids].transpose(0, 2, 1, 3).reshape(-1, kv, D)[:n]
        # the appended rows are the ones this step computed (a rounding of bf16 or E4M3 away)
        assert np.allclose(K[n - T:], kn[at:at + T], rtol=2.0 ** -4, atol=ks * 2.0 ** -9) and np.allclose(V[n - T:], vn[at:at + T], rtol=2.0 ** -4, atol=vs * 2.0 ** -9)
        qq = glue.bf16_to_f32(bf16_to_np(q[at:at + T])).astype(np.float64).reshape(T, heads, D)
        wo, wl_, a, ds = paged.attention(qq, K, V, s.scale, s.causal)
        go = glue.bf16_to_f32(bf16_to_np(o[at:at + T])).astype(np.float64).reshape(T, heads, D)
        es = (ds * (D + 4) * 2 * U)[..., None]
        assert (np.abs(go - wo) <= 2.0 ** -8 * np.abs(wo) + a * (2 * es + 2.0 ** -10 + 2.0 ** -18) + 1e-38).all()
        at += T
    # refusals before anything is launched
    for change in (dict(heads=s.heads + 1), dict(cache=None)):
        st = s.fresh()
        if "heads" in change:
            st[3].c.heads += 1
        else:
            st[3].c.slots = None
        with pytest.raises(rd.RudderError):
            s.fused(st, 1)
        torch.cuda.synchronize()
        assert torch.isnan(st[6]).all().item() and torch.isnan(st[0][0]).all().item()


def test_graphs_that_share_a_workspace_and_replays(rd):
    """Two captured steps with one workspace, replayed in turn with new inputs in the same buffers."""
    a = Step(rd, old=[900, 20], new=[4, 4], heads=4, kv=1, D=64, seed=1)
    b = Step(rd, old=[5, 60, 2000], new=[2, 1, 6], heads=4, kv=2, D=128, seed=2, causal=True)
    sa, sb = a.fresh(), b.fresh()
    ws = sa[5] if sa[5].numel() >= sb[5].numel() else sb[5]
    ws.fill_(0xFF)                                                  # NaN everywhere: nothing may be read before it is written
    sa, sb = (*sa[:5], ws, sa[6]), (*sb[:5], ws, sb[6])
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        a.fused(sa, 0), b.fused(sb, 0)                             # first use outside of capture
    torch.cuda.synchronize()
    graphs = []
    for s, st in ((a, sa), (b, sb)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            s.fused(st, 1)
        graphs.append(g)
    for round_ in range(3):
        for s in (a, b):
            s.X.copy_(torch.randn(s.X.shape, device="cuda").to(torch.bfloat16))
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for s, st in ((a, sa), (b, sb)):
            got = [t.clone() for t in (*st[0], st[2], st[6])]
            ys, q, o, lse, out = s.one_by_one(1)
            torch.cuda.synchronize()
            for x, y in zip(got, (*ys, lse, out)):
                assert torch.equal(x, y), round_
    last, where = rd.rudder_device_status()
    assert last == 0, (last, where)


def test_two_streams_at_once(rd):
    steps = [Step(rd, old=[1500, 33], new=[3, 8], heads=4, kv=2, D=64, seed=s) for s in (5, 6)]
    states = [s.fresh() for s in steps]
    streams = [torch.cuda.Stream() for _ in steps]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, st, q in zip(steps, states, streams):
            s.fused(st, 1, stream=q)
    torch.cuda.synchronize()
    for s, st in zip(steps, states):
        ys, _, _, lse, out = s.one_by_one(1)
        assert torch.equal(st[2], lse) and torch.equal(st[6], out)


def test_workspace_of_its_own_on_a_side_stream(rd):
    """Attention without a workspace argument on a side stream: the scratch is dropped while the kernels run."""
    s = Step(rd, old=[4000], new=[8], heads=8, kv=2, D=64, seed=8)
    rd.rudder_page_tables(s.tables)
    q = torch.randn((8, 512), device="cuda").to(torch.bfloat16)
    side = torch.cuda.Stream()
    outs = []
    torch.cuda.synchronize()
    for _ in range(4):
        o = torch.zeros_like(q)
        side.wait_stream(torch.cuda.current_stream())
        rd.rudder_attention_paged(rd.AttentionArgs(q, 8, s.cache, s.table, s.lens, 0.125, o, max_q=8), stream=side)
        with torch.cuda.stream(side):
            torch.empty(4 << 20, dtype=torch.uint8, device="cuda").fill_(255)      # what the allocator hands out next
        outs.append(o)
    torch.cuda.synchronize()
    assert all(torch.equal(outs[0], o) for o in outs) and outs[0].abs().sum().item() > 0
