"""Cases of the operators for many requests that continue one context: forking, releasing and compacting the pages of a
paged key-value cache, attention of requests that share a prefix, and low-rank adapters of many requests beside a shared
projection.

A case is run in its plain form (elementary torch operations in 32 bits, rounded once at the end) or, where ``own`` is
true, through the framework's entry points.  ``exact`` gives the same outputs from the definitions in 64 bits.
"""
import math
import random

import torch

own = False

DEV = "cuda"


# ---------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # eight candidate action chunks branch off one short context, two layers: the latency of a fork
        {"name": "fork_8_of_one", "op": "fork", "parents": 1, "children": 8, "low": 333, "top": 333, "page": 16, "layers": 2, "Hkv": 16, "D": 128, "fmt": "bf16", "lens": 1},
        # sixteen candidates each of four robots, over the video context of a 2048-wide block (4480 tokens), twelve layers
        {"name": "fork_64_of_four", "op": "fork", "parents": 4, "children": 64, "low": 4000, "top": 4480, "page": 64, "layers": 12, "Hkv": 16, "D": 128, "fmt": "bf16", "lens": 2},
        # those eight candidates and their parent: all but one go
        {"name": "release_9", "op": "release", "B": 9, "page": 16, "top": 349, "shared": 320, "drop": 7, "lens": 3},
        # a full server of 512 requests of up to 16384 tokens, groups of which share their beginnings; a third of them ends
        {"name": "release_512", "op": "release", "B": 512, "page": 64, "top": 16384, "shared": 2048, "drop": 171, "lens": 4},
        # a small pool with holes, one layer: the plan and the renaming are all there is
        {"name": "compact_9", "op": "compact", "B": 9, "page": 16, "top": 349, "shared": 320, "spare": 40, "layers": 1, "Hkv": 4, "D": 64, "fmt": "bf16", "lens": 5},
        # a pool of 48 requests out of which a third of the pages has gone, an 8-bit cache of four layers
        {"name": "compact_48_e4m3", "op": "compact", "B": 48, "page": 32, "top": 16384, "shared": 1024, "spare": 1500, "layers": 4, "Hkv": 8, "D": 128, "fmt": "e4m3", "lens": 6},
        # eight candidates, one new token each, over a short common context: latency
        {"name": "shared_8_short", "op": "attn", "groups": 1, "each": 8, "T": 1, "Hq": 16, "Hkv": 16, "D": 128, "page": 16, "fmt": "bf16", "low": 320, "top": 320, "own": 16,
         "causal": False, "ragged_q": False, "lens": 7},
        # 32 candidate chunks of 16 action rows over the video context of the 2048-wide block: one denoising step of all of them
        {"name": "shared_32x16_chunks", "op": "attn", "groups": 1, "each": 32, "T": 16, "Hq": 16, "Hkv": 16, "D": 128, "page": 64, "fmt": "bf16", "low": 4416, "top": 4416, "own": 80,
         "causal": False, "ragged_q": False, "lens": 8},
        # four long contexts with sixteen continuations each, grouped heads, an 8-bit cache, ragged on both sides and causal
        {"name": "shared_64_long_e4m3", "op": "attn", "groups": 4, "each": 16, "T": 3, "Hq": 32, "Hkv": 8, "D": 128, "page": 32, "fmt": "e4m3", "low": 8000, "top": 32768, "own": 1024,
         "causal": True, "ragged_q": True, "lens": 9},
        # one row with an adapter of rank 16 beside the QKV projection of the 2048-wide block
        {"name": "lora_1row", "op": "lora", "M": 1, "K": 2048, "N": 6144, "R": 16, "adapters": 8, "run": 1, "lens": 10},
        # 64 requests with adapters of their own, ranks mixed up to 64, some without one
        {"name": "lora_64rows", "op": "lora", "M": 64, "K": 2048, "N": 6144, "R": 64, "adapters": 40, "run": 1, "lens": 11},
        # the video context with the adapters of four robots, beside the up projection
        {"name": "lora_4416rows", "op": "lora", "M": 4416, "K": 2048, "N": 8192, "R": 64, "adapters": 4, "run": 1104, "lens": 12},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["fork", "release", "compact", "attn", "attn", "lora", "lora"])
    lens = rng.randrange(1 << 30)
    if op == "fork":
        parents, layers, D = _spread(rng, 1, 8), rng.choice([1, 2, 3, 6]), rng.choice([64, 128, 256])
        top = _spread(rng, 2, 4480)
        return {"op": op, "parents": parents, "children": _spread(rng, 1, 64), "low": rng.choice([1, max(1, top // 2), top]), "top": top, "page": rng.choice([8, 16, 32, 64]),
                "layers": layers, "Hkv": rng.choice([1, 2, 4, 8]), "D": D, "fmt": rng.choice(["bf16", "e4m3"]), "lens": lens}
    if op == "release":
        B, top = _spread(rng, 1, 512), _spread(rng, 8, 16384)
        return {"op": op, "B": B, "page": rng.choice([16, 32, 64, 128]), "top": top, "shared": rng.choice([0, top // 8, top // 2]), "drop": rng.randint(0, B), "lens": lens}
    if op == "compact":
        B, top = _spread(rng, 1, 48), _spread(rng, 8, 8192)
        return {"op": op, "B": B, "page": rng.choice([16, 32, 64]), "top": top, "shared": rng.choice([0, top // 8, top // 2]), "spare": _spread(rng, 1, 500),
                "layers": rng.choice([1, 2, 3]), "Hkv": rng.choice([1, 2, 4, 8]), "D": rng.choice([64, 128]), "fmt": rng.choice(["bf16", "e4m3"]), "lens": lens}
    if op == "attn":
        D = rng.choice([64, 128, 128, 256])
        Hkv, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 1, 2, 3, 4, 8])
        groups, each, T = _spread(rng, 1, 6), _spread(rng, 1, 32), rng.choice([1, 1, 1, 2, _spread(rng, 1, 16)])
        top = _spread(rng, 16, max(32, min(32768, 10 ** 8 // (groups * Hkv * D))))
        return {"op": op, "groups": groups, "each": each, "T": T, "Hq": Hkv * group, "Hkv": Hkv, "D": D, "page": rng.choice([8, 16, 32, 64, 128]),
                "fmt": rng.choice(["bf16", "bf16", "e4m3"]), "low": rng.choice([0, top // 2, top]), "top": top, "own": T + _spread(rng, 1, 512), "causal": rng.random() < 0.5,
                "ragged_q": rng.random() < 0.5, "lens": lens}
    M = _spread(rng, 1, 2048)
    return {"op": op, "M": M, "K": 128 * max(1, round(_spread(rng, 128, 4096) / 128)), "N": 64 * max(1, round(_spread(rng, 64, 8192) / 64)),
            "R": rng.choice([8, 16, 16, 32, 64, 128]), "adapters": rng.choice([1, 2, 3, 8, 20]), "run": rng.choice([1, 1, 3, 16, 77, 500]), "lens": lens}


# ------------------------------------------------------------------- sizes that belong to the case and not to the seed
def _pages(total, page):
    return [-(-t // page) for t in total]


def _fork_lens(case):
    """(length of each parent, which parent each child branches off)."""
    rng = random.Random(case["lens"])
    lens = [rng.randint(case["low"], case["top"]) for _ in range(case["parents"])]
    return lens, [rng.randrange(case["parents"]) if i >= case["parents"] else i for i in range(case["children"])]


def _pool_lens(case):
    """(length of each request, how many of its first pages it shares with the request in front, requests that end)."""
    rng = random.Random(case["lens"])
    B, page = case["B"], case["page"]
    total = [_spread(rng, 1, case["top"]) for _ in range(B)]
    same = [0] + [min(case["shared"] // page, total[b] // page, total[b - 1] // page) if rng.random() < 0.7 else 0 for b in range(1, B)]
    drop = sorted(rng.sample(range(B), case["drop"])) if case["op"] == "release" else []
    return total, same, drop


def _attn_lens(case):
    """(prefix of each group, whole pages; length of each request; its new tokens)."""
    rng = random.Random(case["lens"])
    prefix = [rng.randint(case["low"], case["top"]) // case["page"] * case["page"] for _ in range(case["groups"])]
    total, new = [], []
    for g in range(case["groups"]):
        for _ in range(case["each"]):
            n = rng.randint(1, case["T"]) if case["ragged_q"] else case["T"]
            new.append(n)
            total.append(prefix[g] + rng.randint(n, case["own"]))
    return prefix, total, new


def _lora_rows(case):
    """(adapter of each row, -1 for none; rank of each adapter)."""
    rng = random.Random(case["lens"])
    n, R = case["adapters"], case["R"]
    ranks = [R if n == 1 or rng.random() < 0.5 else rng.choice([R, max(1, R // 2), max(1, R // 4), rng.randint(1, R)]) for _ in range(n)]
    rows = []
    while len(rows) < case["M"]:
        a = rng.randrange(n) if rng.random() < 0.9 or not rows else -1
        rows += [a] * case["run"]
    return rows[:case["M"]], ranks


# --------------------------------------------------------------------------------------------- inputs
def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 64 + salt)
    return g


def _int(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device=DEV)


def _kind(case):
    return torch.bfloat16 if case["fmt"] == "bf16" else torch.float8_e4m3fn


def _bits(t):
    return t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.uint8)


def _caches(case, g, n_pages):
    """The layers' keys and values: one random page after another, every layer and page other numbers."""
    shape = (n_pages, case["Hkv"], case["page"], case["D"])
    return [torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16).to(_kind(case)) for _ in range(2 * case["layers"])]


def prepare(case, seed):
    st = {"case": case}
    globals()["_prepare_" + case["op"]](case, seed, st)
    if own:
        import paper_2609_39056_b200 as rd

        st["rd"] = rd
        globals()["_plan_" + case["op"]](case, st, rd)
    return st


def _prepare_fork(case, seed, st):
    lens, src = _fork_lens(case)
    P, n, page = case["parents"], case["children"], case["page"]
    g = _gen(seed, 1)
    pages = _pages(lens, page)
    have, width = sum(pages), max(pages) + 1
    order = torch.randperm(have + n + 3, generator=g, device=DEV).to(torch.int32)
    table = torch.full((P + n, width), -1, dtype=torch.int32, device=DEV)
    held = torch.arange(width, device=DEV)[None, :] < _int(pages)[:, None]
    table[:P][held] = order[:have]
    st.update(table=table, lens=_int(lens + [0] * n), src=_int(src), dst=_int(list(range(P, P + n))), free=order[have:].contiguous(),
              copies=torch.zeros((n, 3), dtype=torch.int32, device=DEV), used=torch.zeros(1, dtype=torch.int32, device=DEV), caches=_caches(case, g, order.numel()))


def _pool(case, g, extra):
    """(page table with shared beginnings, lengths, number of pages): the requests' pages lie all over a pool with `extra` unused ones."""
    total, same, _ = _pool_lens(case)
    pages = _pages(total, case["page"])
    B, width = case["B"], max(pages)
    fresh = [p - s for p, s in zip(pages, same)]
    n_pages = sum(fresh) + extra
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    col = torch.arange(width, device=DEV)[None, :]
    own_part = (col >= _int(same)[:, None]) & (col < _int(pages)[:, None])
    table = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
    table[own_part] = order[:sum(fresh)]
    row = torch.arange(B, device=DEV)[:, None].expand(B, width)
    first = torch.where(col >= _int(same)[:, None], row, -1).cummax(0).values            # the request that a shared page came from
    table = torch.where(col < _int(pages)[:, None], table.gather(0, first.clamp(min=0)), table)
    return table.contiguous(), _int(total), n_pages


def _prepare_release(case, seed, st):
    _, _, drop = _pool_lens(case)
    table, lens, n_pages = _pool(case, _gen(seed, 2), 11)
    st.update(table=table, lens=lens, drop=_int(drop), refs=torch.zeros(n_pages, dtype=torch.int32, device=DEV),
              free=torch.zeros(n_pages, dtype=torch.int32, device=DEV), n_free=torch.zeros(1, dtype=torch.int32, device=DEV))


def _prepare_compact(case, seed, st):
    g = _gen(seed, 3)
    table, lens, n_pages = _pool(case, g, case["spare"])
    st.update(table=table, lens=lens, new_table=torch.zeros_like(table), remap=torch.zeros(n_pages, dtype=torch.int32, device=DEV),
              copies=torch.zeros((n_pages // 2, 3), dtype=torch.int32, device=DEV), n_copies=torch.zeros(1, dtype=torch.int32, device=DEV),
              n_live=torch.zeros(1, dtype=torch.int32, device=DEV), caches=_caches(case, g, n_pages))


def _prepare_attn(case, seed, st):
    prefix, total, new = _attn_lens(case)
    Hq, Hkv, D, page, G, each = (case[k] for k in ("Hq", "Hkv", "D", "page", "groups", "each"))
    g = _gen(seed, 4)
    lead = [p // page for p in prefix]
    behind = [n - lead[b // each] for b, n in enumerate(_pages(total, page))]
    n_pages, width = sum(lead) + sum(behind) + 2, max(_pages(total, page))
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    col = torch.arange(width, device=DEV)[None, :]
    first = torch.full((G, width), -1, dtype=torch.int32, device=DEV)
    first[col < _int(lead)[:, None]] = order[:sum(lead)]
    table = first.repeat_interleave(each, 0)
    start = _int(lead).repeat_interleave(each)[:, None]
    table[(col >= start) & (col < start + _int(behind)[:, None])] = order[sum(lead):sum(lead) + sum(behind)]
    k = torch.randn((n_pages, Hkv, page, D), generator=g, device=DEV).to(_kind(case))
    v = torch.randn((n_pages, Hkv, page, D), generator=g, device=DEV).to(_kind(case))
    # what stands behind a request's last token in its last page has never been written: NaN
    b = torch.tensor([i for i, t in enumerate(total) if t % page], dtype=torch.int64, device=DEV)
    if b.numel():
        t = _int(total).long()[b]
        last = table[b, t // page].long()
        mask = (torch.arange(page, device=DEV)[None, :] >= (t % page)[:, None])[:, None, :, None].expand(-1, Hkv, -1, D)
        for c in (_bits(k), _bits(v)):
            part = c[last]
            part[mask] = 0x7FC0 if case["fmt"] == "bf16" else 0x7F
            c[last] = part
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    M = starts[-1]
    st.update(k=k, v=v, table=table.contiguous(), total=_int(total), ks=None, vs=None, scale=1.0 / math.sqrt(D), group_starts=_int([i * each for i in range(G + 1)]),
              prefix=_int(prefix), prefix_rows=_int([i * each for i in range(G)]), longest=max(prefix), most=max(t - prefix[b // each] for b, t in enumerate(total)),
              group_q=max(sum(new[i * each:(i + 1) * each]) for i in range(G)), starts=_int(starts), new=_int(new),
              rows=_int([b * case["T"] + i for b, n in enumerate(new) for i in range(n)], torch.int64))        # of [B, T], the real ones
    if case["fmt"] == "e4m3":
        st["ks"] = torch.exp(0.3 * torch.randn(Hkv, generator=g, device=DEV))
        st["vs"] = torch.exp(0.3 * torch.randn(Hkv, generator=g, device=DEV))
    st["q"] = torch.randn((M, Hq * D), generator=g, device=DEV).to(torch.bfloat16)
    st["o"] = torch.zeros((M, Hq * D), dtype=torch.bfloat16, device=DEV)
    st["lse"] = torch.zeros((M, Hq), dtype=torch.float32, device=DEV)


def _prepare_lora(case, seed, st):
    rows, ranks = _lora_rows(case)
    M, K, N, R, n = (case[k] for k in ("M", "K", "N", "R", "adapters"))
    g = _gen(seed, 5)
    st["x"] = torch.randn((M, K), generator=g, device=DEV).to(torch.bfloat16)
    st["base"] = torch.randn((M, N), generator=g, device=DEV).to(torch.bfloat16)                    # what the shared projection gave
    st["a"] = (torch.randn((n, R, K), generator=g, device=DEV) / math.sqrt(K)).to(torch.bfloat16)   # behind an adapter's rank: an older one's
    st["b"] = (torch.randn((n, N, R), generator=g, device=DEV) / math.sqrt(R)).to(torch.bfloat16)
    st["scales"] = 0.5 + torch.rand(n, generator=g, device=DEV)
    st["ranks"], st["rows"] = _int(ranks), _int(rows)
    st["y"] = torch.empty((M, N), dtype=torch.bfloat16, device=DEV)


# ------------------------------------------------------------- what a user's program builds once beside its buffers
def _plan_fork(case, st, rd):
    st["args"] = rd.PageForkArgs(st["table"], st["lens"], case["page"], st["src"], st["dst"], st["free"], st["used"], copies=st["copies"])
    st["list"] = _plan_caches(st, rd)


def _plan_caches(st, rd):
    c = st["caches"]
    return rd.PagedCaches([rd.PagedCache(c[i], c[i + 1]) for i in range(0, len(c), 2)])


def _plan_release(case, st, rd):
    st["args"] = rd.PageReleaseArgs(st["table"], st["lens"], case["page"], st["refs"], st["free"], st["n_free"], drop=st["drop"])


def _plan_compact(case, st, rd):
    st["args"] = rd.PageCompactArgs(st["table"], st["lens"], case["page"], st["new_table"], st["remap"], st["copies"], st["n_copies"], st["n_live"])
    st["list"] = _plan_caches(st, rd)


def _plan_attn(case, st, rd):
    cache = rd.PagedCache(st["k"], st["v"], st["ks"], st["vs"])
    attn = rd.AttentionArgs(st["q"], case["Hq"], cache, st["table"], st["total"], st["scale"], st["o"], q_starts=st["starts"] if case["ragged_q"] else None,
                            max_q=case["T"], causal=case["causal"], lse=st["lse"])
    st["args"] = rd.SharedAttentionArgs(attn, st["group_starts"], st["prefix"], st["prefix_rows"], st["group_q"])
    st["ws"] = torch.empty(rd.rudder_attention_shared_workspace_bytes(st["args"]) + 256, dtype=torch.uint8, device=DEV)


def _plan_lora(case, st, rd):
    st["args"] = rd.LoraArgs(st["x"], st["a"], st["b"], st["ranks"], st["scales"], st["rows"], st["base"], st["y"])
    st["ws"] = torch.empty(rd.rudder_lora_workspace_bytes(st["args"]) + 256, dtype=torch.uint8, device=DEV)


# ------------------------------------------------------------------------------------------- one pass
def run(state):
    case = state["case"]
    if own:
        rd, op = state["rd"], case["op"]
        if op == "fork":
            rd.rudder_page_fork(state["args"], state["list"])
            return _fork_out(state)
        if op == "release":
            rd.rudder_page_release(state["args"])
            return {"lens": state["lens"], "refs": state["refs"], "free": state["free"], "n_free": state["n_free"]}
        if op == "compact":
            rd.rudder_page_compact(state["args"], state["list"])
            return _compact_out(state)
        if op == "attn":
            rd.rudder_attention_shared(state["args"], state["ws"])
            return {"o": state["o"], "lse": state["lse"]}
        rd.rudder_lora(state["args"], state["ws"])
        return {"y": state["y"]}
    return _PLAIN[case["op"]](case, state)


def _fork_out(st):
    return {"table": st["table"], "lens": st["lens"], "copies": st["copies"], "used": st["used"], "caches": st["caches"]}


def _compact_out(st):
    return {"table": st["new_table"], "remap": st["remap"], "copies": st["copies"], "n_copies": st["n_copies"], "n_live": st["n_live"], "caches": st["caches"]}


def _move(cache, src, dst, keep):
    """Tokens [0, keep) of pages `src` to pages `dst`."""
    c = _bits(cache)
    old, page = c[dst], cache.shape[2]
    c[dst] = torch.where((torch.arange(page, device=DEV)[None, :] < keep[:, None])[:, None, :, None], c[src], old)


def _plain_fork(case, st):
    page, table, src, dst = case["page"], st["table"], st["src"].long(), st["dst"].long()
    lens = st["lens"].long()[src]
    full, rest = lens // page, lens % page
    part = rest > 0
    col = torch.arange(table.shape[1], device=DEV)[None, :]
    take = (part.long().cumsum(0) - part.long()).clamp(max=st["free"].numel() - 1)
    fresh = st["free"][take]
    old = table[src]
    rows = torch.where(col < full[:, None], old, table[dst])
    rows = torch.where(part[:, None] & (col == full[:, None]), fresh[:, None], rows)
    table[dst] = rows
    st["lens"][dst] = lens.int()
    at = old.gather(1, full.clamp(max=table.shape[1] - 1)[:, None])[:, 0]
    st["copies"].copy_(torch.stack([torch.where(part, at, -1), torch.where(part, fresh, -1), rest.int()], 1))
    st["used"].copy_(part.sum(0, keepdim=True))
    i = torch.nonzero(part).flatten()
    for c in st["caches"]:
        _move(c, at[i].long(), fresh[i].long(), rest[i])
    return _fork_out(st)


def _references(table, lens, page, n_pages):
    held = torch.arange(table.shape[1], device=DEV)[None, :] < ((lens.long() + page - 1) // page)[:, None]
    return torch.bincount(table[held].long(), minlength=n_pages)


def _plain_release(case, st):
    st["lens"][st["drop"].long()] = 0
    refs = _references(st["table"], st["lens"], case["page"], st["refs"].numel())
    free = torch.nonzero(refs == 0).flatten().int()
    st["refs"].copy_(refs)
    st["free"].fill_(-1)
    st["free"][:free.numel()] = free
    st["n_free"].fill_(free.numel())
    return {"lens": st["lens"], "refs": st["refs"], "free": st["free"], "n_free": st["n_free"]}


def _plain_compact(case, st):
    page, n_pages = case["page"], st["remap"].numel()
    live = _references(st["table"], st["lens"], page, n_pages) > 0
    n_live = live.sum()
    at = torch.arange(n_pages, device=DEV)
    src, dst = torch.nonzero(live & (at >= n_live)).flatten(), torch.nonzero(~live & (at < n_live)).flatten()
    to = torch.where(live, at, -1)
    to[src] = dst
    held = torch.arange(st["table"].shape[1], device=DEV)[None, :] < ((st["lens"].long() + page - 1) // page)[:, None]
    st["new_table"].copy_(torch.where(held, to[st["table"].long().clamp(min=0)].int(), st["table"]))
    st["remap"].copy_(to)
    st["copies"][:src.numel()] = torch.stack([src, dst, torch.full_like(src, page)], 1).int()
    st["n_copies"].fill_(src.numel())
    st["n_live"].copy_(n_live[None])
    for c in st["caches"]:
        _bits(c)[dst] = _bits(c)[src]
    return _compact_out(st)


def _gathered(cache, pages, scale):
    """[n, Hkv, pages x page, D] of the given pages [n, pages], in 32 bits."""
    x = cache[pages.long().clamp(min=0)].float().permute(0, 2, 1, 3, 4)
    x = x.reshape(pages.shape[0], cache.shape[1], -1, cache.shape[3])
    return x if scale is None else x * scale[None, :, None, None]


def _softmax_part(q, k, v, sees, scale):
    """(maximum, sum, weighted values) of rows [n, Hkv, r, D] over keys [n, Hkv, L, D]; sees [n, 1, r or 1, L]."""
    s = torch.where(sees, torch.matmul(q, k.transpose(-1, -2)) * scale, float("-inf"))
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(torch.isfinite(m), m, 0.0))
    used = sees.any(-2)[..., None]                                         # [n, 1, L, 1]
    return m, p.sum(-1, keepdim=True), torch.matmul(p, torch.where(used, v, 0.0))


def _plain_attn(case, st):
    G, each, T, Hq, Hkv, D, page = (case[k] for k in ("groups", "each", "T", "Hq", "Hkv", "D", "page"))
    B, group = G * each, Hq // Hkv
    t = torch.arange(T, device=DEV)
    row = st["starts"][:B, None].long() + t                                # [B, T]
    q = st["q"][row.clamp(max=st["q"].shape[0] - 1)].float().reshape(B, T, Hkv, group, D).permute(0, 2, 1, 3, 4)       # [B, Hkv, T, group, D]
    # the prefix once for all rows of a group
    P = max(1, -(-st["longest"] // page))
    kp, vp = _gathered(st["k"], st["table"][::each, :P], st["ks"]), _gathered(st["v"], st["table"][::each, :P], st["vs"])
    qg = q.reshape(G, each, Hkv, T * group, D).transpose(1, 2).reshape(G, Hkv, -1, D)
    live = torch.arange(P * page, device=DEV) < st["prefix"][:, None]      # [G, L]
    m1, z1, o1 = (x.reshape(G, Hkv, each, T * group, -1).transpose(1, 2).reshape(B, Hkv, T * group, -1)
                  for x in _softmax_part(qg, kp, vp, live[:, None, None, :], st["scale"]))
    # what stands behind it, a request at a time
    S = -(-st["most"] // page)
    lead = (st["prefix"] // page).repeat_interleave(each).long()
    at = (lead[:, None] + torch.arange(S, device=DEV)).clamp(max=st["table"].shape[1] - 1)
    pages = st["table"].gather(1, at)
    ks, vs = _gathered(st["k"], pages, st["ks"]), _gathered(st["v"], pages, st["vs"])
    j = torch.arange(S * page, device=DEV)
    n = (st["total"] - st["prefix"].repeat_interleave(each))[:, None, None]
    sees = j < n
    if case["causal"]:
        sees = sees & (j <= n - st["new"][:, None, None] + t[:, None])
    sees = sees.expand(B, T, S * page).repeat_interleave(group, 1)[:, None]
    m2, z2, o2 = _softmax_part(q.reshape(B, Hkv, T * group, D), ks, vs, sees, st["scale"])
    m = torch.maximum(m1, m2)
    m0 = torch.where(torch.isfinite(m), m, 0.0)
    a, b = torch.exp(m1 - m0), torch.exp(m2 - m0)
    z = z1 * a + z2 * b
    o = (o1 * a + o2 * b) / torch.where(z > 0, z, 1.0)
    lse = (m0 + torch.log(z))[..., 0]
    o = o.reshape(B, Hkv, T, group, D).permute(0, 2, 1, 3, 4).reshape(B * T, Hq * D)[st["rows"]].to(torch.bfloat16)
    return {"o": o, "lse": lse.reshape(B, Hkv, T, group).permute(0, 2, 1, 3).reshape(B * T, Hq)[st["rows"]]}


def _plain_lora(case, st):
    K, N, R, n = case["K"], case["N"], case["R"], case["adapters"]
    used = torch.arange(R, device=DEV)[None, :] < st["ranks"][:, None]                              # [n, R]
    a = torch.where(used[..., None], st["a"].float(), 0.0).reshape(n * R, K)
    b = torch.where(used[:, None, :], st["b"].float(), 0.0) * st["scales"][:, None, None]
    h = torch.matmul(st["x"].float(), a.t()).reshape(-1, n, R)
    h = torch.where((st["rows"][:, None] == torch.arange(n, device=DEV))[..., None], h, 0.0)
    y = torch.matmul(h.reshape(-1, n * R), b.transpose(1, 2).reshape(n * R, N))
    return {"y": (st["base"].float() + y).to(torch.bfloat16)}


_PLAIN = {"fork": _plain_fork, "release": _plain_release, "compact": _plain_compact, "attn": _plain_attn, "lora": _plain_lora}


# ---------------------------------------------------------------------------------------------- work
def work(case):
    op = case["op"]
    if op == "fork":
        lens, src = _fork_lens(case)
        token = 2 * case["layers"] * case["Hkv"] * case["D"] * (2 if case["fmt"] == "bf16" else 1)
        rest, full = sum(lens[s] % case["page"] for s in src), sum(lens[s] // case["page"] for s in src)
        return {"bytes": 2 * token * rest + 8 * full + 36 * len(src), "flops": 0}
    if op in ("release", "compact"):
        total, same, drop = _pool_lens(case)
        pages = _pages(total, case["page"])
        entries = sum(p for b, p in enumerate(pages) if b not in set(drop))
        n_pages = sum(pages) - sum(same) + (11 if op == "release" else case["spare"])
        if op == "release":
            return {"bytes": 4 * entries + 8 * n_pages + 4 * case["B"], "flops": 0}
        live = n_pages - case["spare"]
        moved = live * (n_pages - live) / n_pages                          # as many as lie behind the live ones' number, on average
        page = 2 * case["layers"] * case["Hkv"] * case["page"] * case["D"] * (2 if case["fmt"] == "bf16" else 1)
        return {"bytes": 2 * page * moved + 8 * entries + 4 * n_pages + 12 * moved + 4 * case["B"], "flops": 0}
    if op == "attn":
        prefix, total, new = _attn_lens(case)
        Hq, Hkv, D, page, each = (case[k] for k in ("Hq", "Hkv", "D", "page", "each"))
        size = 2 if case["fmt"] == "bf16" else 1
        behind = [t - prefix[b // each] for b, t in enumerate(total)]
        pages = sum(p // page for p in prefix) + sum(_pages(behind, page))
        return {"bytes": 2 * size * Hkv * D * (sum(prefix) + sum(behind)) + 4 * pages + sum(new) * Hq * (4 * D + 4) + 8 * len(total),
                "flops": 4 * D * Hq * sum(t * n for t, n in zip(total, new))}
    rows, ranks = _lora_rows(case)
    M, K, N = case["M"], case["K"], case["N"]
    return {"bytes": 2 * M * K + 4 * M * N + 4 * M + sum(2 * ranks[a] * (K + N) for a in set(rows) if a >= 0), "flops": 2 * (K + N) * sum(ranks[a] for a in rows if a >= 0)}


# ----------------------------------------------------------------------------------- in 64 bits, one piece at a time
def exact(case, seed):
    st = {"case": case}
    globals()["_prepare_" + case["op"]](case, seed, st)
    return globals()["_exact_" + case["op"]](case, st)


def _exact_fork(case, st):
    lens, src = _fork_lens(case)
    caches = [c.double() for c in st["caches"]]
    table, free, taken = st["table"].tolist(), st["free"].tolist(), 0
    for s in src:
        full, rest = divmod(lens[s], case["page"])
        if rest:
            for c in caches:
                c[free[taken], :, :rest] = c[table[s][full], :, :rest]
            taken += 1
    return {"table": None, "lens": None, "copies": None, "used": None, "caches": caches}


def _exact_release(case, st):
    return None                                                   # whole numbers


def _exact_compact(case, st):
    page = case["page"]
    alive = set()
    for row, n in zip(st["table"].tolist(), st["lens"].tolist()):
        alive.update(row[:-(-n // page)])
    n = len(alive)
    holes, movers = sorted(set(range(n)) - alive), sorted(p for p in alive if p >= n)
    caches = []
    for c in st["caches"]:
        c = c.double()
        c[_int(holes, torch.int64)] = c[_int(movers, torch.int64)]
        caches.append(c)
    return {"table": None, "remap": None, "copies": None, "n_copies": None, "n_live": None, "caches": caches}


def _exact_attn(case, st):
    Hq, Hkv, D, page, group = case["Hq"], case["Hkv"], case["D"], case["page"], case["Hq"] // case["Hkv"]
    _, total, new = _attn_lens(case)
    o = torch.zeros(st["o"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(st["lse"].shape, float("-inf"), dtype=torch.float64, device=DEV)
    first = 0
    for b, (n, t) in enumerate(zip(total, new)):
        pages = st["table"][b, :-(-n // page)].long()
        for h in range(Hkv if n else 0):
            k = st["k"][pages, h].double().reshape(-1, D)[:n]
            v = st["v"][pages, h].double().reshape(-1, D)[:n]
            if st["ks"] is not None:
                k, v = k * st["ks"][h].double(), v * st["vs"][h].double()
            q = st["q"][first:first + t, h * group * D:(h + 1) * group * D].double().reshape(t, group, D)
            s = torch.einsum("tgd,ld->tgl", q, k) * st["scale"]
            if case["causal"]:
                gone = torch.arange(n, device=DEV)[None, :] > (n - t) + torch.arange(t, device=DEV)[:, None]
                s = s.masked_fill(gone[:, None, :], float("-inf"))
            z = torch.logsumexp(s, -1)
            o[first:first + t, h * group * D:(h + 1) * group * D] = torch.einsum("tgl,ld->tgd", torch.exp(s - z[..., None]), v).reshape(t, group * D)
            lse[first:first + t, h * group:(h + 1) * group] = z
        first += t
    return {"o": o, "lse": lse}


def _exact_lora(case, st):
    rows, ranks = _lora_rows(case)
    y = st["base"].double()
    for a in sorted(set(rows) - {-1}):
        m = _int([i for i, r in enumerate(rows) if r == a], torch.int64)
        h = st["x"][m].double() @ st["a"][a, :ranks[a]].double().t()
        y[m] += st["scales"][a].double() * (h @ st["b"][a, :, :ranks[a]].double().t())
    return {"y": y}
