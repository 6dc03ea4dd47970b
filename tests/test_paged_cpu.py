"""Refusals of the paged-cache operators (host checks, before anything is launched: no GPU needed) and pins of their
plain counterparts in the oracle."""
import ctypes

import numpy as np
import pytest

from oracle import glue, paged

FAKE = 0x10000      # never dereferenced


@pytest.fixture(scope="module")
def rd():
    from paper_2609_39056_b200 import build
    build.build()
    import paper_2609_39056_b200 as rd
    rd.lib()
    return rd


def cache_c(rd, **kw):
    d = dict(k=FAKE, v=FAKE, format=rd.CACHE_BF16, n_pages=8, page_size=16, heads=2, head_dim=128, page_stride=2 * 16 * 128, head_stride=16 * 128,
             token_stride=128, k_scale=None, v_scale=None)
    d.update(kw)
    return rd._PagedCache(**d)


def table_c(rd, **kw):
    d = dict(old_lens=FAKE, new_lens=FAKE, B=3, page_size=16, free_pages=FAKE, n_free=4, page_table=FAKE, ld_table=8, max_pages=8, slots=FAKE,
             positions=FAKE, capacity=5, starts=FAKE, used=FAKE)
    d.update(kw)
    return rd._PageTableArgs(**d)


def qk_c(rd, cache=None, **kw):
    d = dict(X=FAKE, ldx=1024, M=3, heads=4, kv_heads=2, head_dim=128, q_weight=FAKE, k_weight=FAKE, eps=1e-6, cos=FAKE, sin=FAKE, n_pos=64, rot=128,
             style=rd.ROPE_HALF, positions=FAKE, Q=FAKE, ldq=512, K=FAKE, ldk=256, slots=None)
    d.update(kw)
    a = rd._QkArgs(**d)
    if cache is not None:
        a.cache = ctypes.pointer(cache)
    return a


def attn_c(rd, cache, **kw):
    d = dict(Q=FAKE, ldq=512, M=4, heads=4, page_table=FAKE, ld_table=8, max_pages=8, kv_lens=FAKE, q_starts=None, B=4, max_q=1, causal=0, scale=0.1,
             O=FAKE, ldo=512, lse=None)
    d.update(kw)
    a = rd._AttentionArgs(**d)
    if cache is not None:
        a.cache = ctypes.pointer(cache)
    return a


@pytest.mark.parametrize("kw,want", [
    (dict(old_lens=None), "ARG"), (dict(new_lens=None), "ARG"), (dict(page_table=None), "ARG"), (dict(slots=None), "ARG"), (dict(positions=None), "ARG"),
    (dict(starts=None), "ARG"), (dict(used=None), "ARG"), (dict(free_pages=None), "ARG"), (dict(n_free=-1), "ARG"), (dict(page_size=0), "SHAPE"),
    (dict(page_size=24), "SHAPE"), (dict(page_size=2048), "SHAPE"), (dict(B=0), "SHAPE"), (dict(B=8193), "SHAPE"), (dict(max_pages=0), "SHAPE"),
    (dict(ld_table=7), "SHAPE"), (dict(capacity=0), "SHAPE"), (dict(capacity=1 << 30), "SHAPE")])
def test_page_tables_refusals(rd, kw, want):
    assert rd.lib().rudder_page_tables(ctypes.byref(table_c(rd, **kw)), None) == getattr(rd, "ERR_" + want)


@pytest.mark.parametrize("kw,want", [
    (dict(X=None), "ARG"), (dict(Q=None), "ARG"), (dict(K=None), "ARG"), (dict(slots=FAKE), "ARG"), (dict(eps=-1.0), "ARG"), (dict(eps=float("nan")), "ARG"),
    (dict(style=2), "UNSUPPORTED"), (dict(M=0), "SHAPE"), (dict(heads=0), "SHAPE"), (dict(kv_heads=0), "SHAPE"), (dict(head_dim=96), "SHAPE"),
    (dict(rot=8), "SHAPE"), (dict(rot=144), "SHAPE"), (dict(rot=-16), "SHAPE"), (dict(cos=None), "ARG"), (dict(sin=None), "ARG"),
    (dict(positions=None), "ARG"), (dict(n_pos=0), "ARG"), (dict(X=FAKE + 2), "ALIGN"), (dict(ldx=1020), "ALIGN"), (dict(ldx=1016), "ALIGN"),
    (dict(ldq=504), "ALIGN"), (dict(Q=FAKE + 8), "ALIGN"), (dict(ldk=248), "ALIGN"), (dict(q_weight=FAKE + 4), "ALIGN"), (dict(cos=FAKE + 4), "ALIGN")])
def test_qk_refusals(rd, kw, want):
    assert rd.lib().rudder_qk_norm_rope(ctypes.byref(qk_c(rd, **kw)), None) == getattr(rd, "ERR_" + want)


BAD_CACHES = [
    (dict(k=None), "ARG"), (dict(v=None), "ARG"), (dict(n_pages=0), "ARG"), (dict(format=2), "UNSUPPORTED"), (dict(page_size=12), "SHAPE"),
    (dict(page_size=0), "SHAPE"), (dict(k=FAKE + 8), "ALIGN"), (dict(v=FAKE + 8), "ALIGN"), (dict(token_stride=132), "ALIGN"), (dict(head_stride=64), "ALIGN"),
    (dict(page_stride=-128), "ALIGN"), (dict(token_stride=0), "ALIGN"), (dict(page_stride=0), "ALIGN"), (dict(format=1, token_stride=136), "ALIGN")]


@pytest.mark.parametrize("kw,want", BAD_CACHES)
def test_cache_refusals(rd, kw, want):
    c = cache_c(rd, **kw)
    L = rd.lib()
    assert L.rudder_qk_norm_rope(ctypes.byref(qk_c(rd, c, K=None, slots=FAKE)), None) == getattr(rd, "ERR_" + want)
    assert L.rudder_attention_paged(ctypes.byref(attn_c(rd, c)), FAKE, 1 << 30, None) == getattr(rd, "ERR_" + want)


def test_qk_cache_shape_and_targets(rd):
    L = rd.lib()
    assert L.rudder_qk_norm_rope(ctypes.byref(qk_c(rd, cache_c(rd, heads=4), K=None, slots=FAKE)), None) == rd.ERR_SHAPE
    assert L.rudder_qk_norm_rope(ctypes.byref(qk_c(rd, cache_c(rd, head_dim=64), K=None, slots=FAKE)), None) == rd.ERR_SHAPE
    assert L.rudder_qk_norm_rope(ctypes.byref(qk_c(rd, cache_c(rd), slots=FAKE)), None) == rd.ERR_ARG            # both K and a cache
    assert L.rudder_qk_norm_rope(ctypes.byref(qk_c(rd, cache_c(rd), K=None)), None) == rd.ERR_ARG                # a cache without slots
    assert L.rudder_qk_norm_rope(None, None) == rd.ERR_ARG


@pytest.mark.parametrize("kw,want", [
    (dict(Q=None), "ARG"), (dict(O=None), "ARG"), (dict(page_table=None), "ARG"), (dict(kv_lens=None), "ARG"), (dict(scale=float("nan")), "ARG"),
    (dict(scale=float("inf")), "ARG"), (dict(B=0), "SHAPE"), (dict(max_q=0), "SHAPE"), (dict(heads=3), "SHAPE"), (dict(heads=0), "SHAPE"), (dict(M=0), "SHAPE"),
    (dict(M=3), "SHAPE"), (dict(max_pages=0), "SHAPE"), (dict(ld_table=4), "SHAPE"), (dict(max_q=1 << 20), "SHAPE"),
    (dict(max_pages=1 << 28, ld_table=1 << 28), "SHAPE"), (dict(ldq=504), "ALIGN"), (dict(ldo=516), "ALIGN"), (dict(Q=FAKE + 2), "ALIGN"), (dict(O=FAKE + 2), "ALIGN")])
def test_attention_refusals(rd, kw, want):
    assert rd.lib().rudder_attention_paged(ctypes.byref(attn_c(rd, cache_c(rd), **kw)), FAKE, 1 << 30, None) == getattr(rd, "ERR_" + want)


def test_attention_workspace(rd):
    L = rd.lib()
    c = cache_c(rd)
    a = attn_c(rd, c)
    need = L.rudder_attention_workspace_bytes(ctypes.byref(a))
    assert need > 0
    assert L.rudder_attention_paged(ctypes.byref(a), None, need, None) == rd.ERR_WORKSPACE
    assert L.rudder_attention_paged(ctypes.byref(a), FAKE, need - 1, None) == rd.ERR_WORKSPACE
    assert L.rudder_attention_paged(ctypes.byref(a), FAKE + 128, need, None) == rd.ERR_WORKSPACE
    assert L.rudder_attention_workspace_bytes(None) == 0
    assert L.rudder_attention_workspace_bytes(ctypes.byref(attn_c(rd, None))) == 0
    assert L.rudder_attention_workspace_bytes(ctypes.byref(attn_c(rd, c, heads=3))) == 0


def test_linear_a16_and_block_refuse_null(rd):
    L = rd.lib()
    assert L.rudder_linear_a16(None, FAKE, 128, 1, None, FAKE, 128, None) == rd.ERR_ARG
    assert L.rudder_block_cached(None, None, None, None, 1, None, 0, None, 0, None) == rd.ERR_ARG
    assert L.rudder_block_cached_workspace_bytes(None, None, 1) == 0


# ---- pins of the oracle -----------------------------------------------------------------------------------------------

def test_oracle_page_tables_by_hand():
    table = np.full((2, 3), -1, np.int32)
    table[0, 0] = 7
    t, slots, pos, starts, used = paged.page_tables(np.array([3, 0]), np.array([2, 5]), np.array([9, 4, 2]), table, 4, 9)
    # request 0: tokens 3, 4 -> page 7 place 3, new page 9 place 0; request 1: tokens 0..4 -> pages 4, 2
    assert t.tolist() == [[7, 9, -1], [4, 2, -1]] and starts.tolist() == [0, 2, 7] and used == 3
    assert slots.tolist() == [31, 36, 16, 17, 18, 19, 8, -1, -1] and pos.tolist() == [3, 4, 0, 1, 2, 3, 4, -1, -1]


@pytest.mark.parametrize("D", [64, 128, 256])
def test_oracle_qk_against_fp64(D):
    rng = np.random.default_rng(D)
    x = glue.bf16_to_f32(glue.f32_to_bf16((rng.standard_normal((5, 4 * D)) * 2).astype(np.float32)))
    w = (1 + 0.1 * rng.standard_normal(D)).astype(np.float32)
    ang = rng.uniform(0, 6, (9, D // 2))
    c, s = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
    pos = np.array([0, 8, 3, 3, 5])
    for pairs in (False, True):
        q, k, v = paged.qk_norm_rope(x, 2, 1, D, w, w, 1e-6, c, s, D, pairs, pos)
        h = x.reshape(5, 4, D)[:, :3].astype(np.float64)
        y = h / np.sqrt((h ** 2).mean(-1, keepdims=True) + 1e-6) * w
        z = y[..., 0::2] + 1j * y[..., 1::2] if pairs else y[..., :D // 2] + 1j * y[..., D // 2:]
        z = z * (c + 1j * s.astype(np.float64))[pos][:, None]
        want = np.stack([z.real, z.imag], -1).reshape(5, 3, D) if pairs else np.concatenate([z.real, z.imag], -1)
        # some 16 roundings of at most 2^-24 on values below 2 max |y|
        assert np.abs(np.concatenate([q, k], 1) - want).max() <= 40 * 2.0 ** -24 * np.abs(y).max()
        assert np.array_equal(v[:, 0], x.reshape(5, 4, D)[:, 3])


def test_oracle_attention_special_cases():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((3, 2, 64)), rng.standard_normal((5, 1, 64)), rng.standard_normal((5, 1, 64))
    o, lse, _, _ = paged.attention(0 * q, k, v, 1.0, False)
    assert np.allclose(o, v.mean(0)) and np.allclose(lse, np.log(5))                 # equal scores: the mean
    o, lse, _, _ = paged.attention(q, k[:1], v[:1], 0.3, False)
    assert np.allclose(o, v[0]) and np.allclose(lse[..., None], 0.3 * q @ k[0, 0][:, None])   # one key: its value
    o, lse, _, _ = paged.attention(q, k[:2], v[:2], 0.3, True)                         # three rows, two keys: the first sees none
    assert (o[0] == 0).all() and np.isneginf(lse[0]).all() and np.allclose(o[1], v[0])
    o, lse, _, _ = paged.attention(q, k[:0], v[:0], 0.3, False)
    assert (o == 0).all() and np.isneginf(lse).all()


def test_oracle_linear_a16_by_hand():
    codes = np.array([[0x1F, 0x70]], np.uint8)                                       # -1, 1, 0, 7
    y, s = paged.linear_a16(np.array([[1.0, 2.0, 3.0, 4.0]]), codes, np.array([[0.5, 2.0]]), np.array([1.0, 2.0, 1.0, 0.5]), np.array([10.0]))
    assert y.tolist() == [[10 + 0.5 * (-1 + 4) + 2.0 * 14]] and s.tolist() == [[0.5 * 5 + 28]]
    y, _ = paged.linear_a16(np.array([[1.0, 2.0, 3.0, 4.0]]), np.array([[0x91, 0x7A]], np.uint8), np.array([[1.0]]), np.ones(4), None, 2.0)
    assert y.tolist() == [[2 * (0.5 - 1.0 - 3.0 + 24.0)]]
