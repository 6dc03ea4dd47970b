"""Page tables, query / key pass and attention captured back to back, nothing between them: each kernel starts while the one in front
of it still runs and reads what that one writes (table, slots, positions, starts, keys, values)."""
import numpy as np
import pytest
import torch

from test_gpu_paged import cuda, rd, status_clean  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("B,new_top,heads,kv,D", [(3, 1, 8, 2, 128), (200, 3, 2, 1, 64), (5, 40, 2, 2, 128), (40, 20, 1, 1, 256)])
def test_tables_append_and_attention_in_one_graph(rd, B, new_top, heads, kv, D, fmt):  # noqa: F811
    page, top = 16, 700
    rng = np.random.default_rng(B + D)
    width = -(-(top + new_top) // page)
    n_pages, M = B * width, B * new_top
    kind = torch.bfloat16 if fmt == "bf16" else torch.float8_e4m3fn
    g = torch.Generator(device="cuda")
    g.manual_seed(B)
    k0, v0 = (torch.randn((n_pages, kv, page, D), generator=g, device="cuda").to(kind) for _ in range(2))
    kc, vc = k0.clone(), v0.clone()
    cache = rd.PagedCache(kc, vc)
    old, new, lens = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(3))
    free = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    table = torch.zeros((B, width), dtype=torch.int32, device="cuda")
    slots, pos = torch.zeros(M, dtype=torch.int64, device="cuda"), torch.zeros(M, dtype=torch.int32, device="cuda")
    starts, used = torch.zeros(B + 1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    X = torch.zeros((M, (heads + 2 * kv) * D), dtype=torch.bfloat16, device="cuda")
    ang = torch.rand((top + new_top, D // 2), generator=g, device="cuda") * 6
    Q, O = (torch.zeros((M, heads * D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lse = torch.zeros((M, heads), device="cuda")
    tables = rd.PageTableArgs(old, new, free, table, page, slots, pos, starts, used)
    qk = rd.QkArgs(X, heads, kv, D, None, None, 1e-6, torch.cos(ang), torch.sin(ang), rd.ROPE_HALF, pos, Q, cache=cache, slots=slots)
    att = rd.AttentionArgs(Q, heads, cache, table, lens, D ** -0.5, O, q_starts=starts, max_q=new_top, causal=True, lse=lse)
    ws = torch.empty(rd.rudder_attention_workspace_bytes(att) + 256, dtype=torch.uint8, device="cuda")

    def inputs():
        o, n = rng.integers(0, top + 1, B), rng.integers(0, new_top + 1, B)
        held = -(-o // page)
        ids = rng.permutation(n_pages)
        t = np.full((B, width), -1, np.int32)
        at = 0
        for b in range(B):
            t[b, :held[b]] = ids[at:at + held[b]]
            at += held[b]
        rest = np.resize(ids[at:], n_pages)                         # (the list is longer than what is taken)
        for dst, src in ((old, o), (new, n), (lens, o + n), (table, t), (free, rest)):
            dst.copy_(cuda(src.astype(np.int32)))
        kc.copy_(k0), vc.copy_(v0), O.zero_(), lse.zero_(), Q.zero_()
        X.copy_(torch.randn(X.shape, generator=g, device="cuda").to(torch.bfloat16))

    def step(between):
        rd.rudder_page_tables(tables)
        between()
        rd.rudder_qk_norm_rope(qk)
        between()
        rd.rudder_attention_paged(att, ws)

    inputs()
    step(torch.cuda.synchronize)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(lambda: None)
    outs = (table, slots, pos, starts, used, Q, kc.view(torch.uint8), vc.view(torch.uint8), O, lse)
    for _ in range(6):
        inputs()
        saved = [t.clone() for t in (table, kc, vc)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        for t, s in zip((table, kc, vc), saved):
            t.copy_(s)
        O.zero_(), lse.zero_(), Q.zero_()
        step(torch.cuda.synchronize)                                # one at a time
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outs))
        assert (O.abs().sum().item() > 0) == (starts[B].item() > 0)      # (a step may have no new token at all)
    status_clean(rd)
