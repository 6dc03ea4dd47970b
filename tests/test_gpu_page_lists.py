"""Free lists shared by several calls, on the GPU: forks in a row that go by what is taken already, and lists that run out."""
import numpy as np
import pytest
import torch

from oracle import shared
from test_gpu_paged import rd, status_clean  # noqa: F401  (rd: the fixture)
from test_gpu_shared import i32, layers, pool, words

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("per,page,top,n_layers", [(3, 16, 60, 1), (40, 64, 700, 9)])
def test_three_forks_in_a_row_go_by_the_sum(rd, per, page, top, n_layers):
    """`taken` is what all calls before have used since the list was made, added up on the device: no page is handed out twice."""
    rng = np.random.default_rng(per)
    parents = 4
    table, lens, n_pages = pool(rng, parents, page, top, share=0, spare=3 * per + 4)
    lens[:] = np.maximum(lens, 1)
    lens[lens % page == 0] -= 1                                    # every parent has a started page
    lens = np.maximum(lens, 1).astype(np.int32)
    for b in range(parents):
        for c in range(-(-int(lens[b]) // page)):
            assert table[b, c] >= 0
    free = np.setdiff1d(np.arange(n_pages), table)[::-1].copy().astype(np.int32)
    T0 = np.concatenate([table, np.full((3 * per, table.shape[1]), -5, np.int32)])
    L0 = np.concatenate([lens, np.zeros(3 * per, np.int32)])
    caches, handle = layers(rd, n_layers, n_pages, 2, page, 64, "bf16", seed=per)
    before = [words(c) for c in caches]
    T, L, F = i32(T0), i32(L0), i32(free)
    taken, used = i32([0]), i32([77])
    want_t, want_l, at = T0, L0, 0
    for turn in range(3):
        src = rng.integers(0, parents, per).astype(np.int32)
        dst = parents + per * turn + np.arange(per, dtype=np.int32)
        rd.rudder_page_fork(rd.PageForkArgs(T, L, page, i32(src), i32(dst), F, used, taken=taken), handle)
        taken += used
        want_t, want_l, copies, n = shared.fork(want_t, want_l, page, src.tolist(), dst.tolist(), free, None, at)
        at += n
        before = [shared.copy_tokens(b, copies) for b in before]
    assert taken.item() == at == 3 * per
    assert np.array_equal(T.cpu().numpy(), want_t) and np.array_equal(L.cpu().numpy(), want_l)
    started = [int(want_t[b, want_l[b] // page]) for b in range(parents + 3 * per)]
    assert len(set(started)) == len(started)
    for c, b in zip(caches, before):
        assert np.array_equal(words(c), b)
    status_clean(rd)


@pytest.mark.parametrize("n_free", [0, 1, 2, 4, 5])
def test_a_release_list_given_whole_runs_out(rd, n_free):
    """rudder_page_release leaves -1 behind the last free page; a call that is given all entries records that it met one."""
    page, n_pages = 4, 9
    held = n_pages - n_free
    table = np.full((2, 12), -1, np.int32)
    table[1, :held] = np.arange(held)
    T, L = i32(table), i32([0, held * page])
    refs, free, n = (torch.zeros(k, dtype=torch.int32, device="cuda") for k in (n_pages, n_pages, 1))
    rd.rudder_page_release(rd.PageReleaseArgs(T, L, page, refs, free, n))
    assert n.item() == n_free
    new = 15                                                       # four pages
    slots, pos = torch.zeros(16, dtype=torch.int64, device="cuda"), torch.zeros(16, dtype=torch.int32, device="cuda")
    starts, used = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    rd.rudder_page_tables(rd.PageTableArgs(L, i32([new, 0]), free, T, page, slots, pos, starts, used))
    got = slots.cpu().numpy()
    want = [int(free[t // page]) * page + t % page if t // page < n_free else -1 for t in range(new)] + [-1]
    assert got.tolist() == want and used.item() == 4
    assert rd.rudder_device_status() == ((rd.OK, 0) if n_free >= 4 else (rd.ERR_ARG, rd.NO_PAGES))
