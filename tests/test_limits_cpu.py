"""Sizes whose index arithmetic would leave 32 bits are refused on the host (no GPU needed)."""
import ctypes

from tests.test_paged_cpu import FAKE, rd  # noqa: F401  (rd: the fixture)
from tests.test_shared_cpu import fork_c


def test_fork_columns(rd):
    """A warp steps over a row's columns 32 at a time: as in the other operators on pages, 2^30 of them at most."""
    assert rd.lib().rudder_page_fork(ctypes.byref(fork_c(rd, page_size=1, max_pages=(1 << 30) + 1, ld_table=1 << 31)), None, 0, None) == rd.ERR_SHAPE
    assert rd.lib().rudder_page_fork(ctypes.byref(fork_c(rd, page_size=1, max_pages=(1 << 31) - 1, ld_table=1 << 31)), None, 0, None) == rd.ERR_SHAPE
