"""Free lists shared by several calls, on the GPU: lists that run out."""
import numpy as np
import pytest
import torch

from test_gpu_paged import rd  # noqa: F401  (rd: the fixture)
from test_gpu_shared import i32

pytestmark = pytest.mark.gpu


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
