"""Sizes whose index arithmetic would leave 32 bits are refused on the host (no GPU needed)."""
import ctypes

import pytest

from tests.test_paged_cpu import FAKE, rd  # noqa: F401  (rd: the fixture)
from tests.test_shared_cpu import fork_c, lora_c

OVER = (1 << 30) + 8


def test_fork_columns(rd):
    """A warp steps over a row's columns 32 at a time: as in the other operators on pages, 2^30 of them at most."""
    assert rd.lib().rudder_page_fork(ctypes.byref(fork_c(rd, page_size=1, max_pages=(1 << 30) + 1, ld_table=1 << 31)), None, 0, None) == rd.ERR_SHAPE
    assert rd.lib().rudder_page_fork(ctypes.byref(fork_c(rd, page_size=1, max_pages=(1 << 31) - 1, ld_table=1 << 31)), None, 0, None) == rd.ERR_SHAPE


@pytest.mark.parametrize("kw", [dict(M=(1 << 30) + 1), dict(M=(1 << 31) - 1), dict(K=OVER, ldx=OVER, lda=OVER, a_stride=16 * OVER),
                                dict(N=OVER, ldy=OVER, ld_base=OVER, b_stride=16 * OVER), dict(K=(1 << 31) - 8, ldx=1 << 31, lda=1 << 31), dict(N=(1 << 31) - 8, ldy=1 << 31, ld_base=1 << 31)])
def test_lora_sizes(rd, kw):
    assert rd.lib().rudder_lora_workspace_bytes(ctypes.byref(lora_c(rd, **kw))) == 0
    assert rd.lib().rudder_lora(ctypes.byref(lora_c(rd, **kw)), FAKE, 1 << 62, None) == rd.ERR_SHAPE


def test_lora_largest_sizes_are_planned(rd):
    """At the limits the plan's numbers stay inside 32 bits: the workspace has room for a row of sums at least, and for a list of the rows."""
    big = 1 << 30
    for kw, least in ((dict(M=big), big * 16 * 4 + big * 4), (dict(K=big, ldx=big, lda=big), 3 * 16 * 4), (dict(N=big, ldy=big, ld_base=big), 3 * 16 * 4)):
        assert least <= rd.lib().rudder_lora_workspace_bytes(ctypes.byref(lora_c(rd, **kw))) < 1 << 40
