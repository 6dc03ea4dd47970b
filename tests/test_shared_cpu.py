"""Refusals of the operators for many requests that continue one context (host checks, before anything is launched: no GPU needed) and pins of
their plain counterparts in the oracle."""
import ctypes

import numpy as np
import pytest

from oracle import shared
from tests.test_paged_cpu import BAD_CACHES, FAKE, attn_c, cache_c, rd  # noqa: F401  (rd: the fixture)


def fork_c(rd, **kw):
    d = dict(page_table=FAKE, ld_table=8, max_pages=8, lens=FAKE, B=5, page_size=16, src=FAKE, dst=FAKE, fork_lens=None, n=3, free_pages=FAKE, n_free=4, taken=None,
             copies=None, used=FAKE)
    d.update(kw)
    return rd._PageForkArgs(**d)


def release_c(rd, **kw):
    d = dict(page_table=FAKE, ld_table=8, max_pages=8, lens=FAKE, B=5, page_size=16, drop=FAKE, n_drop=2, n_pages=9, refs=FAKE, free_pages=FAKE, n_free=FAKE)
    d.update(kw)
    return rd._PageReleaseArgs(**d)


def compact_c(rd, **kw):
    d = dict(page_table=FAKE, ld_table=8, max_pages=8, lens=FAKE, B=5, page_size=16, n_pages=8, new_table=FAKE + 4096, ld_new=8, remap=FAKE, copies=FAKE, n_copies=FAKE,
             n_live=FAKE)
    d.update(kw)
    return rd._PageCompactArgs(**d)


def lora_c(rd, **kw):
    d = dict(X=FAKE, ldx=64, M=3, K=64, A=FAKE, a_stride=16 * 64, lda=64, B=FAKE, b_stride=128 * 16, ldb=16, N=128, R=16, n_adapters=4, ranks=FAKE, scales=FAKE,
             adapters=FAKE, base=FAKE, ld_base=128, Y=FAKE + 4096, ldy=128)
    d.update(kw)
    return rd._LoraArgs(**d)


def shared_c(rd, cache, attn=None, **kw):
    d = dict(group_starts=FAKE, prefix_lens=FAKE, prefix_rows=FAKE, n_groups=2, table_rows=4, group_q=2)
    d.update(kw)
    s = rd._SharedAttentionArgs(**d)
    s.attn = attn_c(rd, cache, **(attn or {}))
    return s


def caches_c(rd, *kws):
    return (rd._PagedCache * len(kws))(*(cache_c(rd, **k) for k in kws))


def want_of(rd, name):
    return getattr(rd, "ERR_" + name)


COMMON = [(dict(page_table=None), "ARG"), (dict(lens=None), "ARG"), (dict(page_size=24), "SHAPE"), (dict(page_size=2048), "SHAPE"), (dict(B=0), "SHAPE"),
          (dict(max_pages=0), "SHAPE"), (dict(ld_table=7), "SHAPE")]


@pytest.mark.parametrize("kw,want", COMMON + [
    (dict(src=None), "ARG"), (dict(dst=None), "ARG"), (dict(used=None), "ARG"), (dict(free_pages=None), "ARG"), (dict(n_free=-1), "ARG"), (dict(n=0), "SHAPE"),
    (dict(n=8193), "SHAPE"), (dict(B=8193), "SHAPE")])
def test_fork_refusals(rd, kw, want):
    assert rd.lib().rudder_page_fork(ctypes.byref(fork_c(rd, **kw)), None, 0, None) == want_of(rd, want)


@pytest.mark.parametrize("kw,want", COMMON + [
    (dict(refs=None), "ARG"), (dict(free_pages=None), "ARG"), (dict(n_free=None), "ARG"), (dict(drop=None), "ARG"), (dict(n_drop=-1), "ARG"), (dict(n_pages=0), "SHAPE"),
    (dict(n_pages=(1 << 30) + 1), "SHAPE"), (dict(B=(1 << 20) + 1), "SHAPE"), (dict(max_pages=(1 << 30) + 1, ld_table=1 << 31), "SHAPE")])
def test_release_refusals(rd, kw, want):
    assert rd.lib().rudder_page_release(ctypes.byref(release_c(rd, **kw)), None) == want_of(rd, want)


@pytest.mark.parametrize("kw,want", COMMON + [
    (dict(new_table=None), "ARG"), (dict(remap=None), "ARG"), (dict(copies=None), "ARG"), (dict(n_copies=None), "ARG"), (dict(n_live=None), "ARG"), (dict(n_pages=0), "SHAPE"),
    (dict(ld_new=7), "SHAPE"), (dict(new_table=FAKE, ld_new=9), "SHAPE"), (dict(max_pages=(1 << 30) + 1, ld_table=1 << 31, ld_new=1 << 31), "SHAPE")])
def test_compact_refusals(rd, kw, want):
    assert rd.lib().rudder_page_compact(ctypes.byref(compact_c(rd, **kw)), None, 0, None) == want_of(rd, want)


def test_compact_refuses_another_pool(rd):
    c = caches_c(rd, {})
    assert rd.lib().rudder_page_compact(ctypes.byref(compact_c(rd, n_pages=7)), c, 1, None) == rd.ERR_SHAPE


@pytest.mark.parametrize("kw,want", BAD_CACHES + [(dict(page_size=32, head_stride=32 * 128, page_stride=2 * 32 * 128), "SHAPE")])
def test_layers_refusals(rd, kw, want):
    for kws in ([kw], [{}, kw]):
        assert rd.lib().rudder_page_fork(ctypes.byref(fork_c(rd)), caches_c(rd, *kws), len(kws), None) == want_of(rd, want)
        if "page_size" not in kw or len(kws) > 1:
            assert rd.lib().rudder_page_copy(ctypes.byref(rd._PageCopyArgs(FAKE, None, 4)), caches_c(rd, *kws), len(kws), None) == want_of(rd, want)


@pytest.mark.parametrize("kw", [dict(heads=1), dict(head_dim=64), dict(n_pages=9), dict(token_stride=256, head_stride=32 * 128), dict(page_stride=3 * 16 * 128), dict(format=1)])
def test_layers_of_one_geometry(rd, kw):
    assert rd.lib().rudder_page_copy(ctypes.byref(rd._PageCopyArgs(FAKE, None, 4)), caches_c(rd, {}, kw), 2, None) == rd.ERR_SHAPE


def test_layers_limits(rd):
    many = caches_c(rd, *[{}] * 129)
    copy = lambda n, c, k: rd.lib().rudder_page_copy(ctypes.byref(rd._PageCopyArgs(FAKE, None, n)), c, k, None)  # noqa: E731
    assert copy(4, many, 129) == rd.ERR_SHAPE
    assert copy(4, None, 1) == rd.ERR_ARG and copy(4, many, 0) == rd.ERR_ARG and copy(4, many, -1) == rd.ERR_ARG and copy(0, many, 1) == rd.ERR_SHAPE
    assert copy((1 << 31) // 4, many, 1) == rd.ERR_SHAPE                     # 2 x 1 layer x 2 heads x n at 2^31
    assert rd.lib().rudder_page_fork(ctypes.byref(fork_c(rd)), None, 1, None) == rd.ERR_ARG
    assert rd.lib().rudder_page_copy(ctypes.byref(rd._PageCopyArgs(None, None, 4)), many, 1, None) == rd.ERR_ARG


@pytest.mark.parametrize("kw,want", [
    (dict(X=None), "ARG"), (dict(A=None), "ARG"), (dict(B=None), "ARG"), (dict(Y=None), "ARG"), (dict(ranks=None), "ARG"), (dict(scales=None), "ARG"),
    (dict(adapters=None), "ARG"), (dict(M=0), "SHAPE"), (dict(K=60), "SHAPE"), (dict(K=0), "SHAPE"), (dict(N=100), "SHAPE"), (dict(R=12), "SHAPE"), (dict(R=0), "SHAPE"),
    (dict(R=264), "SHAPE"), (dict(n_adapters=0), "SHAPE"), (dict(n_adapters=4097), "SHAPE"), (dict(X=FAKE + 2), "ALIGN"), (dict(ldx=68), "ALIGN"), (dict(ldx=56), "ALIGN"),
    (dict(ldy=120), "ALIGN"), (dict(lda=56), "ALIGN"), (dict(ldb=8), "ALIGN"), (dict(a_stride=1028), "ALIGN"), (dict(b_stride=-8), "ALIGN"), (dict(base=FAKE + 8), "ALIGN"),
    (dict(ld_base=120), "ALIGN"), (dict(base=FAKE + 4096, ld_base=136), "ALIGN")])
def test_lora_refusals(rd, kw, want):
    assert rd.lib().rudder_lora(ctypes.byref(lora_c(rd, **kw)), FAKE, 1 << 30, None) == want_of(rd, want)


@pytest.mark.parametrize("kw,want", [
    (dict(group_starts=None), "ARG"), (dict(prefix_lens=None), "ARG"), (dict(prefix_rows=None), "ARG"), (dict(n_groups=0), "SHAPE"), (dict(table_rows=3), "SHAPE"),
    (dict(group_q=0), "SHAPE"), (dict(attn=dict(M=(1 << 19) + 1, B=1)), "SHAPE"), (dict(attn=dict(Q=None)), "ARG"), (dict(attn=dict(heads=3)), "SHAPE"),
    (dict(attn=dict(scale=float("inf"))), "ARG"), (dict(attn=dict(M=3)), "SHAPE"), (dict(attn=dict(ldo=504)), "ALIGN")])
def test_shared_refusals(rd, kw, want):
    cache = cache_c(rd)
    assert rd.lib().rudder_attention_shared(ctypes.byref(shared_c(rd, cache, **kw)), FAKE, 1 << 30, None) == want_of(rd, want)


@pytest.mark.parametrize("workspace,size", [(None, 1 << 30), (FAKE + 8, 1 << 30), (FAKE, 16)])
def test_workspaces(rd, workspace, size):
    cache = cache_c(rd)
    assert rd.lib().rudder_attention_shared(ctypes.byref(shared_c(rd, cache)), workspace, size, None) == rd.ERR_WORKSPACE
    assert rd.lib().rudder_lora(ctypes.byref(lora_c(rd)), workspace, size, None) == rd.ERR_WORKSPACE
    assert rd.lib().rudder_lora_workspace_bytes(ctypes.byref(lora_c(rd, R=12))) == 0


# ---- the oracle's own pins
def test_oracle_fork_by_hand():
    table = np.array([[7, 3, -1], [-1, -1, -1], [-1, -1, -1], [5, -1, -1]], np.int32)
    lens = np.array([5, 0, 0, 4], np.int32)
    new, ln, copies, used = shared.fork(table, lens, 4, [0, 3], [1, 2], [9, 8], None, 0)
    assert new[1].tolist() == [7, 9, -1] and new[2].tolist() == [5, -1, -1] and ln.tolist() == [5, 5, 4, 4]
    assert copies.tolist() == [[3, 9, 1], [-1, -1, 0]] and used == 1


def test_oracle_fork_leaves_out():
    table = np.array([[7, 3], [-1, -1], [2, -1]], np.int32)
    lens = np.array([5, 0, 2], np.int32)
    # a row that is read, a row taken twice, rows that do not exist, a length that the parent has not got
    new, ln, copies, used = shared.fork(table, lens, 4, [0, 0, 0, 3, 0], [2, 1, 1, 1, -1], [9, 8], [5, 6, 5, 1, 1], 0)
    assert ln.tolist() == [5, 0, 5] and new[2].tolist() == [7, 9] and used == 1
    new, ln, _, _ = shared.fork(table, lens, 4, [0, 2], [2, 1], [9, 8], None, 0)
    assert ln.tolist() == [5, 2, 2] and new[1].tolist() == [9, -1]


def test_oracle_release_and_compact_by_hand():
    table = np.array([[4, 1, 0], [4, 6, -1], [2, -1, -1]], np.int32)
    lens = np.array([5, 8, 1], np.int32)
    ln, refs, free, n = shared.release(table, lens, 4, [2], 8)
    assert ln.tolist() == [5, 8, 0] and refs.tolist() == [0, 1, 0, 0, 2, 0, 1, 0] and free.tolist() == [0, 2, 3, 5, 7, -1, -1, -1] and n == 5
    new, remap, copies, n_live = shared.compact(table, ln, 4, 8)
    assert n_live == 3 and copies.tolist() == [[4, 0, 4], [6, 2, 4]] and remap.tolist() == [-1, 1, -1, -1, 0, -1, 2, -1]
    assert new.tolist() == [[0, 1, 0], [0, 2, -1], [2, -1, -1]]
