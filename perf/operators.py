"""Cases of the serving operators around a paged key-value cache: page tables, query / key norm with rotation, attention
of new tokens over the cache, and 4-bit-weight products of a few rows.

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
        # four robots, one new token each: the bookkeeping of the smallest step
        {"name": "tables_4x1", "op": "tables", "B": 4, "page": 16, "top": 700, "new": 1, "lens": 1},
        # a full server: 512 requests of up to 16384 tokens, chunks of up to 64 new tokens and some idle requests
        {"name": "tables_512_ragged", "op": "tables", "B": 512, "page": 64, "top": 16384, "new": 64, "lens": 2},
        # one action chunk of 16 rows after the QKV linear of a 2048-wide block, written to the cache
        {"name": "qk_16rows", "op": "qk", "M": 16, "Hq": 16, "Hkv": 16, "D": 128, "rot": 128, "style": "half", "page": 16, "fmt": "bf16"},
        # the video context of that block (4096 + 64 + 256 rows) into an 8-bit cache
        {"name": "qk_4416rows_e4m3", "op": "qk", "M": 4416, "Hq": 16, "Hkv": 16, "D": 128, "rot": 128, "style": "half", "page": 64, "fmt": "e4m3"},
        # grouped heads, part of each head turned in neighbouring pairs, an odd number of rows
        {"name": "qk_1021rows_pairs", "op": "qk", "M": 1021, "Hq": 24, "Hkv": 4, "D": 64, "rot": 32, "style": "pairs", "page": 32, "fmt": "bf16"},
        # one new token over a short context: latency
        {"name": "attn_one_short", "op": "attn", "B": 1, "T": 1, "Hq": 16, "Hkv": 16, "D": 128, "page": 16, "fmt": "bf16", "low": 333, "top": 333, "causal": False, "ragged_q": False, "lens": 1},
        # 16 proprio + 48 action rows over the video context of the 2048-wide block: one denoising step
        {"name": "attn_chunk64", "op": "attn", "B": 1, "T": 64, "Hq": 16, "Hkv": 16, "D": 128, "page": 64, "fmt": "bf16", "low": 4480, "top": 4480, "causal": False, "ragged_q": False, "lens": 1},
        # a serving batch with grouped heads and an 8-bit cache, lengths spread from empty to long
        {"name": "attn_batch48_e4m3", "op": "attn", "B": 48, "T": 1, "Hq": 32, "Hkv": 8, "D": 128, "page": 32, "fmt": "e4m3", "low": 0, "top": 16384, "causal": False, "ragged_q": False, "lens": 3},
        # a few new tokens of each request, causal among themselves, ragged on both sides
        {"name": "attn_ragged_causal", "op": "attn", "B": 9, "T": 5, "Hq": 16, "Hkv": 4, "D": 64, "page": 16, "fmt": "bf16", "low": 0, "top": 2501, "causal": True, "ragged_q": True, "lens": 4},
        # four requests with very long contexts
        {"name": "attn_long", "op": "attn", "B": 4, "T": 1, "Hq": 32, "Hkv": 4, "D": 128, "page": 128, "fmt": "bf16", "low": 120000, "top": 131072, "causal": False, "ragged_q": False, "lens": 5},
        # one row (a step embedding) through a square layer with groups of 64
        {"name": "a16_1x2048x2048", "op": "a16", "M": 1, "K": 2048, "N": 2048, "scheme": "w4a8", "group": 64},
        # a small action batch through the down projection of the 2048-wide block, NVFP4 weights
        {"name": "a16_8x8192x2048_nvfp4", "op": "a16", "M": 8, "K": 8192, "N": 2048, "scheme": "nvfp4", "group": 16},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tables", "qk", "attn", "attn", "a16"])
    if op == "tables":
        return {"op": op, "B": _spread(rng, 1, 512), "page": rng.choice([8, 16, 32, 64, 128]), "top": _spread(rng, 8, 16384), "new": _spread(rng, 1, 64),
                "lens": rng.randrange(1 << 30)}
    if op == "qk":
        D = rng.choice([64, 128, 256])
        Hkv = rng.choice([1, 2, 4, 8])
        rot = rng.choice([0, 16, 32, D // 2, D, D])
        return {"op": op, "M": _spread(rng, 1, 4096), "Hq": Hkv * rng.choice([1, 1, 2, 3, 4]), "Hkv": Hkv, "D": D, "rot": rot, "style": rng.choice(["half", "pairs"]),
                "page": rng.choice([8, 16, 32, 64, 128]), "fmt": rng.choice(["bf16", "e4m3"])}
    if op == "attn":
        D = rng.choice([64, 128, 128, 256])
        Hkv = rng.choice([1, 2, 4, 8])
        group = rng.choice([1, 1, 2, 3, 4, 8])
        T = rng.choice([1, 1, 1, 2, _spread(rng, 1, 64)])
        B = _spread(rng, 1, 48)
        top = _spread(rng, 1, max(2, min(65536, 3 * 10 ** 8 // (B * Hkv * D))))
        return {"op": op, "B": B, "T": T, "Hq": Hkv * group, "Hkv": Hkv, "D": D, "page": rng.choice([8, 16, 32, 64, 128]), "fmt": rng.choice(["bf16", "bf16", "e4m3"]),
                "low": rng.choice([0, top // 2, top]), "top": top, "causal": rng.random() < 0.5, "ragged_q": rng.random() < 0.5, "lens": rng.randrange(1 << 30)}
    scheme, group = rng.choice([("w4a8", 64), ("w4a8", 128), ("w4a4", 64), ("w4a8", 0), ("nvfp4", 16)])
    K = 256 * max(1, round(_spread(rng, 256, 8192) / 256))
    return {"op": "a16", "M": rng.choice([1, 1, 2, 3, 5, 8, 13, 16]), "K": K, "N": 64 * max(1, round(_spread(rng, 64, 8192) / 64)),
            "scheme": scheme, "group": group if group else K}


def _lens(case):
    """Lengths that belong to the case (not to the seed): (cached length incl. the new tokens, new tokens) of each request."""
    rng = random.Random(case["lens"])
    B, top = case["B"], case["top"]
    if case["op"] == "tables":
        total = [_spread(rng, 1, top) for _ in range(B)]
        new = [min(t, rng.choice([0, 1, 1, rng.randint(1, case["new"])]) if case["new"] > 1 else case["new"]) for t in total]
        return total, new
    low = case["low"]
    total = [rng.randint(low, top) if low else (0 if rng.random() < 0.1 else _spread(rng, 1, top)) for _ in range(B)]
    new = [rng.randint(1, case["T"]) if case["ragged_q"] else case["T"] for _ in range(B)]
    return total, new


# --------------------------------------------------------------------------------------------- inputs
def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 64 + salt)
    return g


def _pages(total, page):
    return [-(-t // page) for t in total]


def _int(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device=DEV)


def prepare(case, seed):
    st = {"case": case}
    globals()["_prepare_" + case["op"]](case, seed, st)
    if own:
        import paper_2609_39056_b200 as rd

        st["rd"] = rd
        globals()["_plan_" + case["op"]](case, st, rd)
    return st


def _prepare_tables(case, seed, st):
    total, new = _lens(case)
    B, page = case["B"], case["page"]
    old = [t - n for t, n in zip(total, new)]
    width = max(1, max(_pages(total, page)))
    have = sum(_pages(old, page))
    used = sum(_pages(total, page)) - have
    order = torch.randperm(have + used + 9, generator=_gen(seed, 1), device=DEV).to(torch.int32)
    held = torch.arange(width, device=DEV)[None, :] < _int(_pages(old, page))[:, None]
    table = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
    table[held] = order[:have]
    capacity = sum(new) + 3                                       # some rows of padding behind the last request
    st.update(old=_int(old), new=_int(new), free=order[have:].contiguous(), table=table, capacity=capacity,
              slots=torch.empty(capacity, dtype=torch.int64, device=DEV), positions=torch.empty(capacity, dtype=torch.int32, device=DEV),
              starts=torch.empty(B + 1, dtype=torch.int32, device=DEV), used=torch.empty(1, dtype=torch.int32, device=DEV))


def _prepare_qk(case, seed, st):
    M, Hq, Hkv, D, rot, page = (case[k] for k in ("M", "Hq", "Hkv", "D", "rot", "page"))
    g = _gen(seed, 2)
    width = (Hq + 2 * Hkv) * D
    x = torch.randn((M, width), generator=g, device=DEV) * torch.exp(0.5 * torch.randn((1, width), generator=g, device=DEV))
    st["x"] = x.to(torch.bfloat16)
    st["qw"] = 1 + 0.1 * torch.randn(D, generator=g, device=DEV)
    st["kw"] = 1 + 0.1 * torch.randn(D, generator=g, device=DEV)
    st["eps"] = 1e-6
    n_pos = 8192
    if rot:
        freq = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
        angle = torch.arange(n_pos, dtype=torch.float64, device=DEV)[:, None] * freq[None, :]
        st["cos"], st["sin"] = torch.cos(angle).float(), torch.sin(angle).float()
    pos = torch.randint(0, n_pos, (M,), generator=g, device=DEV, dtype=torch.int32)
    n_pages = -(-M // page) + 5
    slots = torch.randperm(n_pages * page, generator=g, device=DEV)[:M].contiguous()
    pad = M // 16                                                 # rows of padding behind the last request
    if pad:
        pos[M - pad:] = -1
        slots[M - pad:] = -1
    st["pos"], st["slots"], st["real"] = pos, slots, M - pad
    shape = (n_pages, Hkv, page, D)
    kind = torch.bfloat16 if case["fmt"] == "bf16" else torch.float8_e4m3fn
    st["k"] = torch.randn(shape, generator=g, device=DEV).to(kind)
    st["v"] = torch.randn(shape, generator=g, device=DEV).to(kind)
    st["ks"] = st["vs"] = None
    if case["fmt"] == "e4m3":
        st["ks"] = 0.02 * torch.exp(0.3 * torch.randn(Hkv, generator=g, device=DEV))
        st["vs"] = 0.02 * torch.exp(0.3 * torch.randn(Hkv, generator=g, device=DEV))
    st["q"] = torch.randn((M, Hq * D), generator=g, device=DEV).to(torch.bfloat16)     # rows of padding keep this


def _prepare_attn(case, seed, st):
    Hq, Hkv, D, page = (case[k] for k in ("Hq", "Hkv", "D", "page"))
    total, new = _lens(case)
    g = _gen(seed, 3)
    pages = _pages(total, page)
    n_pages, width = sum(pages) + 2, max(1, max(pages))
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    held = torch.arange(width, device=DEV)[None, :] < _int(pages)[:, None]
    table = torch.full((case["B"], width), -1, dtype=torch.int32, device=DEV)
    table[held] = order[:sum(pages)]
    shape = (n_pages, Hkv, page, D)
    kind = torch.bfloat16 if case["fmt"] == "bf16" else torch.float8_e4m3fn
    k = torch.randn(shape, generator=g, device=DEV).to(kind)
    v = torch.randn(shape, generator=g, device=DEV).to(kind)
    # what stands behind a request's last token in its last page has never been written: NaN
    b = torch.tensor([i for i, t in enumerate(total) if t % page], dtype=torch.int64, device=DEV)
    if b.numel():
        t = _int(total).long()[b]
        last = table[b, t // page].long()
        dead = torch.arange(page, device=DEV)[None, :] >= (t % page)[:, None]
        mask = dead[:, None, :, None].expand(-1, Hkv, -1, D)
        code = k.view(torch.int16 if case["fmt"] == "bf16" else torch.uint8), v.view(torch.int16 if case["fmt"] == "bf16" else torch.uint8)
        for c in code:
            part = c[last]
            part[mask] = 0x7FC0 if case["fmt"] == "bf16" else 0x7F
            c[last] = part
    st.update(k=k, v=v, table=table, lens=_int(total), ks=None, vs=None, scale=1.0 / math.sqrt(D), longest=max(total))
    if case["fmt"] == "e4m3":
        st["ks"] = torch.exp(0.3 * torch.randn(Hkv, generator=g, device=DEV))
        st["vs"] = torch.exp(0.3 * torch.randn(Hkv, generator=g, device=DEV))
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    M = starts[-1]
    st["starts"], st["new"] = _int(starts), _int(new)
    st["rows"] = _int([b * case["T"] + i for b, n in enumerate(new) for i in range(n)], torch.int64)    # of [B, T], the real ones
    st["q"] = torch.randn((M, Hq * D), generator=g, device=DEV).to(torch.bfloat16)
    st["o"] = torch.zeros((M, Hq * D), dtype=torch.bfloat16, device=DEV)
    st["lse"] = torch.zeros((M, Hq), dtype=torch.float32, device=DEV)


def _prepare_a16(case, seed, st):
    M, K, N, G = case["M"], case["K"], case["N"], case["group"]
    g = _gen(seed, 4)
    st["x"] = torch.randn((M, K), generator=g, device=DEV).to(torch.bfloat16)
    st["dinv"] = torch.exp((torch.rand(K, generator=g, device=DEV) * 2 - 1) * math.log(4.0))
    st["bias"] = 0.1 * torch.randn(N, generator=g, device=DEV)
    if case["scheme"] == "nvfp4":
        st["codes"] = torch.randint(0, 256, (N, K // 2), generator=g, device=DEV, dtype=torch.uint8)
        st["scales"] = (torch.rand((N, K // 16), generator=g, device=DEV) * 200 + 20).to(torch.float8_e4m3fn).view(torch.uint8)
        st["ts"] = torch.full((1,), 5e-5, device=DEV)
    else:
        q = torch.randint(-7, 8, (N, K), generator=g, device=DEV, dtype=torch.int32) & 15
        st["codes"] = (q[:, 0::2] | (q[:, 1::2] << 4)).to(torch.uint8)
        st["scales"] = ((torch.rand((N, K // G), generator=g, device=DEV) + 0.5) * 0.008).to(torch.float16)
        st["ts"] = torch.ones(1, device=DEV)
    st["y"] = torch.empty((M, N), dtype=torch.bfloat16, device=DEV)


# ------------------------------------------------------------- what a user's program builds once beside its buffers
def _plan_tables(case, st, rd):
    st["args"] = rd.PageTableArgs(st["old"], st["new"], st["free"], st["table"], case["page"], st["slots"], st["positions"], st["starts"], st["used"])


def _plan_qk(case, st, rd):
    style = rd.ROPE_HALF if case["style"] == "half" else rd.ROPE_PAIRS
    cache = rd.PagedCache(st["k"], st["v"], st["ks"], st["vs"])
    st["args"] = rd.QkArgs(st["x"], case["Hq"], case["Hkv"], case["D"], st["qw"], st["kw"], st["eps"], st.get("cos"), st.get("sin"), style,
                           st["pos"], st["q"], cache=cache, slots=st["slots"])


def _plan_attn(case, st, rd):
    cache = rd.PagedCache(st["k"], st["v"], st["ks"], st["vs"])
    st["args"] = rd.AttentionArgs(st["q"], case["Hq"], cache, st["table"], st["lens"], st["scale"], st["o"], q_starts=st["starts"] if case["ragged_q"] else None,
                                  max_q=case["T"], causal=case["causal"], lse=st["lse"])
    st["ws"] = torch.empty(rd.rudder_attention_workspace_bytes(st["args"]) + 256, dtype=torch.uint8, device=DEV)


def _plan_a16(case, st, rd):
    scheme = {"w4a8": rd.W4A8_INT, "w4a4": rd.W4A4_INT, "nvfp4": rd.W4A4_NVFP4}[case["scheme"]]
    st["w"] = rd.rudder_weight_import({"codes": st["codes"], "scales": st["scales"], "dinv": st["dinv"], "tensor_scale": st["ts"]},
                                      case["N"], case["K"], scheme, case["group"])


# ------------------------------------------------------------------------------------------- one pass
def run(state):
    case = state["case"]
    if own:
        rd, op = state["rd"], case["op"]
        if op == "tables":
            rd.rudder_page_tables(state["args"])
            return {"table": state["table"], "slots": state["slots"], "positions": state["positions"], "starts": state["starts"], "used": state["used"]}
        if op == "qk":
            rd.rudder_qk_norm_rope(state["args"])
            return {"q": state["q"], "k": state["k"], "v": state["v"]}
        if op == "attn":
            rd.rudder_attention_paged(state["args"], state["ws"])
            return {"o": state["o"], "lse": state["lse"]}
        return {"y": rd.rudder_linear_a16(state["w"], state["x"], state["bias"], state["y"])}
    return _PLAIN[case["op"]](case, state)


def _plain_tables(case, st):
    page, table, old, new = case["page"], st["table"], st["old"].long(), st["new"].long()
    held, want = (old + page - 1) // page, (old + new + page - 1) // page
    need = want - held
    first = need.cumsum(0) - need
    col = torch.arange(table.shape[1], device=DEV)[None, :]
    fresh = (col >= held[:, None]) & (col < want[:, None])
    pick = (first[:, None] + col - held[:, None]).clamp(0, st["free"].numel() - 1)
    out = torch.where(fresh, st["free"][pick], table)
    starts = torch.cat([new.new_zeros(1), new.cumsum(0)])
    token = torch.arange(st["capacity"], device=DEV)
    req = torch.searchsorted(starts, token, right=True) - 1
    real = req < old.numel()
    req = req.clamp(max=old.numel() - 1)
    pos = old[req] + token - starts[req]
    page_id = out[req, torch.where(real, pos, 0) // page].long()
    slots = torch.where(real, page_id * page + pos % page, -1)
    return {"table": out, "slots": slots, "positions": torch.where(real, pos, -1).int(), "starts": starts.int(), "used": need.sum(0, keepdim=True).int()}


def _turn(y, cos, sin, rot, style):
    if rot == 0:
        return y
    a, b = (y[..., :rot // 2], y[..., rot // 2:rot]) if style == "half" else (y[..., 0:rot:2], y[..., 1:rot:2])
    c, s = cos[:, None, :], sin[:, None, :]
    u, w = a * c - b * s, b * c + a * s
    turned = torch.cat([u, w], -1) if style == "half" else torch.stack([u, w], -1).flatten(-2)
    return torch.cat([turned, y[..., rot:]], -1)


def _to_cache(x, like, scale):
    if like.dtype == torch.bfloat16:
        return x.to(torch.bfloat16)
    return (x / scale[None, :, None]).clamp(-448, 448).to(torch.float8_e4m3fn)


def _put(cache, slots, rows):
    """Row i of `rows` [M, Hkv, D] into the cache at slots[i]."""
    page = cache.shape[2]
    bits = torch.int16 if cache.dtype == torch.bfloat16 else torch.uint8
    cache.view(bits)[slots // page, :, slots % page] = rows.view(bits)


def _plain_qk(case, st):
    Hq, Hkv, D, rot, n = case["Hq"], case["Hkv"], case["D"], case["rot"], st["real"]
    x = st["x"][:n].float().reshape(n, Hq + 2 * Hkv, D)
    qk = x[:, :Hq + Hkv]
    w = torch.cat([st["qw"].expand(Hq, D), st["kw"].expand(Hkv, D)])
    y = qk * torch.rsqrt((qk * qk).mean(-1, keepdim=True) + st["eps"]) * w
    at = st["pos"][:n].long()
    y = _turn(y, st["cos"][at] if rot else None, st["sin"][at] if rot else None, rot, case["style"])
    st["q"][:n] = y[:, :Hq].reshape(n, Hq * D).to(torch.bfloat16)
    _put(st["k"], st["slots"][:n], _to_cache(y[:, Hq:], st["k"], st["ks"]))
    _put(st["v"], st["slots"][:n], _to_cache(x[:, Hq + Hkv:], st["v"], st["vs"]))
    return {"q": st["q"], "k": st["k"], "v": st["v"]}


def _gathered(cache, table, scale, page, L):
    P = -(-L // page)
    x = cache[table[:, :P].long().clamp(min=0)].float()                     # [B, P, Hkv, page, D]
    x = x.permute(0, 2, 1, 3, 4).reshape(table.shape[0], cache.shape[1], P * page, cache.shape[3])
    return x if scale is None else x * scale[None, :, None, None]


def _plain_attn(case, st):
    B, T, Hq, Hkv, D, page = (case[k] for k in ("B", "T", "Hq", "Hkv", "D", "page"))
    L = max(1, st["longest"])
    k = _gathered(st["k"], st["table"], st["ks"], page, L)
    v = _gathered(st["v"], st["table"], st["vs"], page, L)
    L = k.shape[2]
    t = torch.arange(T, device=DEV)
    row = st["starts"][:B, None].long() + t                                 # [B, T]
    q = st["q"][row.clamp(max=st["q"].shape[0] - 1)].float().reshape(B, T, Hkv, Hq // Hkv, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, D)
    s = torch.matmul(q, k.transpose(-1, -2)) * st["scale"]                  # [B, Hkv, T * group, L]
    j = torch.arange(L, device=DEV)
    live = j < st["lens"][:, None]                                          # [B, L]
    sees = live[:, None, :].expand(B, T, L)
    if case["causal"]:
        sees = sees & (j <= (st["lens"] - st["new"])[:, None, None] + t[:, None])
    sees = sees[:, None, :, None, :].expand(B, Hkv, T, Hq // Hkv, L).reshape(B, Hkv, -1, L)
    s = torch.where(sees, s, float("-inf"))
    m = s.amax(-1, keepdim=True)
    m0 = torch.where(torch.isfinite(m), m, 0.0)
    p = torch.exp(s - m0)
    z = p.sum(-1, keepdim=True)
    o = torch.matmul(p, torch.where(live[:, None, :, None], v, 0.0)) / torch.where(z > 0, z, 1.0)
    lse = (m0 + torch.log(z))[..., 0]
    o = o.reshape(B, Hkv, T, Hq // Hkv, D).permute(0, 2, 1, 3, 4).reshape(B * T, Hq * D)[st["rows"]].to(torch.bfloat16)
    return {"o": o, "lse": lse.reshape(B, Hkv, T, Hq // Hkv).permute(0, 2, 1, 3).reshape(B * T, Hq)[st["rows"]]}


def _weights(case, st, kind):
    """The weights as numbers of the given type, [N, K], with dinv and the scales applied."""
    c = st["codes"]
    q = torch.stack([c & 15, c >> 4], -1).reshape(case["N"], case["K"])
    if case["scheme"] == "nvfp4":
        grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=kind, device=DEV)
        q, s = grid[q.long()], st["scales"].view(torch.float8_e4m3fn).to(kind) * st["ts"].to(kind)
    else:
        q, s = ((q.to(torch.int8) ^ 8) - 8).to(kind), st["scales"].to(kind)
    return (q.reshape(case["N"], -1, case["group"]) * s[..., None]).reshape(case["N"], case["K"]) * st["dinv"].to(kind)


def _plain_a16(case, st):
    return {"y": (torch.matmul(st["x"].float(), _weights(case, st, torch.float32).t()) + st["bias"]).to(torch.bfloat16)}


_PLAIN = {"tables": _plain_tables, "qk": _plain_qk, "attn": _plain_attn, "a16": _plain_a16}


# ---------------------------------------------------------------------------------------------- work
def work(case):
    op = case["op"]
    if op == "tables":
        total, new = _lens(case)
        page = case["page"]
        used = sum(_pages(total, page)) - sum(_pages([t - n for t, n in zip(total, new)], page))
        n = sum(new) + 3
        return {"bytes": 12 * case["B"] + 8 * used + 12 * n + 4 * case["B"] + 8, "flops": 0}
    if op == "qk":
        M, Hq, Hkv, D, rot = (case[k] for k in ("M", "Hq", "Hkv", "D", "rot"))
        real = M - M // 16
        out = 2 if case["fmt"] == "bf16" else 1
        return {"bytes": real * (2 * D * (Hq + 2 * Hkv) + 2 * D * Hq + 2 * out * D * Hkv) + 12 * M + min(real, 8192) * 4 * rot + 8 * D,
                "flops": real * (Hq + Hkv) * (4 * D + 3 * rot)}
    if op == "attn":
        total, new = _lens(case)
        Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
        size = 2 if case["fmt"] == "bf16" else 1
        pages = sum(_pages(total, case["page"]))
        return {"bytes": 2 * size * Hkv * D * sum(total) + 4 * pages + sum(new) * Hq * (4 * D + 4) + 8 * case["B"],
                "flops": 4 * D * Hq * sum(t * n for t, n in zip(total, new))}
    M, K, N, G = case["M"], case["K"], case["N"], case["group"]
    return {"bytes": N * K // 2 + N * (K // G) * (1 if case["scheme"] == "nvfp4" else 2) + 4 * K + 4 * N + 2 * M * (K + N), "flops": 2 * M * K * N}


# ----------------------------------------------------------------------------------- in 64 bits, one piece at a time
def exact(case, seed):
    st = {"case": case}
    globals()["_prepare_" + case["op"]](case, seed, st)
    return globals()["_exact_" + case["op"]](case, st)


def _exact_tables(case, st):
    return None                                                   # whole numbers


def _exact_qk(case, st):
    M, Hq, Hkv, D, rot, page = (case[k] for k in ("M", "Hq", "Hkv", "D", "rot", "page"))
    x = st["x"].double()
    q, k, v = st["q"].double(), st["k"].double(), st["v"].double()
    rows = torch.nonzero((st["pos"] >= 0)).flatten()
    at = st["pos"].long()[rows]
    slot = st["slots"][rows]
    half = torch.arange(rot // 2, device=DEV)
    one, two = (half, half + rot // 2) if case["style"] == "half" else (2 * half, 2 * half + 1)

    def head(h, w):
        y = x[rows, h * D:(h + 1) * D]
        y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / D + st["eps"]) * w.double()
        if rot:
            c, s = st["cos"].double()[at], st["sin"].double()[at]
            z = y.clone()
            z[:, one] = y[:, one] * c - y[:, two] * s
            z[:, two] = y[:, two] * c + y[:, one] * s
            y = z
        return y

    for h in range(Hq):
        q[rows, h * D:(h + 1) * D] = head(h, st["qw"])
    for h in range(Hkv):
        a, b = head(Hq + h, st["kw"]), x[rows, (Hq + Hkv + h) * D:(Hq + Hkv + h + 1) * D]
        if case["fmt"] == "e4m3":
            a, b = (a / st["ks"][h].double()).clamp(-448, 448), (b / st["vs"][h].double()).clamp(-448, 448)
        k[slot // page, h, slot % page] = a
        v[slot // page, h, slot % page] = b
    return {"q": q, "k": k, "v": v}


def _exact_attn(case, st):
    Hq, Hkv, D, page = (case[k] for k in ("Hq", "Hkv", "D", "page"))
    total, new = _lens(case)
    o = torch.zeros(st["o"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(st["lse"].shape, float("-inf"), dtype=torch.float64, device=DEV)
    first = 0
    for b, (n, t) in enumerate(zip(total, new)):
        for h in range(Hkv if n else 0):
            pages = st["table"][b, :-(-n // page)].long()
            k = st["k"][pages, h].double().reshape(-1, D)[:n]
            v = st["v"][pages, h].double().reshape(-1, D)[:n]
            if st["ks"] is not None:
                k, v = k * st["ks"][h].double(), v * st["vs"][h].double()
            g = Hq // Hkv
            q = st["q"][first:first + t, h * g * D:(h + 1) * g * D].double().reshape(t, g, D)
            s = torch.einsum("tgd,ld->tgl", q, k) * st["scale"]
            if case["causal"]:
                gone = torch.arange(n, device=DEV)[None, :] > (n - t) + torch.arange(t, device=DEV)[:, None]
                s = s.masked_fill(gone[:, None, :], float("-inf"))
            z = torch.logsumexp(s, -1)
            p = torch.where(torch.isfinite(z)[..., None], torch.exp(s - z[..., None]), 0.0)
            o[first:first + t, h * g * D:(h + 1) * g * D] = torch.einsum("tgl,ld->tgd", p, v).reshape(t, g * D)
            lse[first:first + t, h * g:(h + 1) * g] = z
        first += t
    return {"o": o, "lse": lse}


def _exact_a16(case, st):
    y = st["bias"].double().repeat(case["M"], 1)
    x = st["x"].double() * st["dinv"].double()
    N, K, G = case["N"], case["K"], case["group"]
    for n in range(0, N, 1024):
        c = st["codes"][n:n + 1024].int()
        w = torch.empty((c.shape[0], K), dtype=torch.float64, device=DEV)
        for part in (0, 1):
            q = (c >> (4 * part)) & 15
            if case["scheme"] == "nvfp4":
                m, e = (q & 1).double(), ((q >> 1) & 3)
                mag = torch.where(e == 0, m * 0.5, (1 + m / 2) * torch.pow(2.0, e.double() - 1))
                w[:, part::2] = torch.where(q >= 8, -mag, mag)
            else:
                w[:, part::2] = torch.where(q >= 8, q - 16, q).double()
        s = st["scales"][n:n + 1024]
        s = s.view(torch.float8_e4m3fn).double() * st["ts"].double() if case["scheme"] == "nvfp4" else s.double()
        y[:, n:n + 1024] += x @ (w * s.repeat_interleave(G, 1)).t()
    return {"y": y}
