"""rudder_page_fork: arguments that cannot be, refused on the host before anything is launched (no GPU needed)."""
import ctypes

import pytest

from tests.test_paged_cpu import FAKE, cache_c, rd  # noqa: F401  (rd: the fixture)
from tests.test_shared_cpu import fork_c

WORD = 4


def refused(rd, **kw):
    one = cache_c(rd)
    for caches, n in ((None, 0), ((rd._PagedCache * 1)(one), 1)):
        assert rd.lib().rudder_page_fork(ctypes.byref(fork_c(rd, **kw)), caches, n, None) == rd.ERR_ARG


# every array at a place of its own, 64 KB apart
PLACES = {name: FAKE + (i << 16) for i, name in enumerate(("page_table", "lens", "src", "dst", "fork_lens", "free_pages", "taken", "copies", "used"))}
ENTRIES = {"lens": 5, "src": 3, "dst": 3, "fork_lens": 3, "free_pages": 4, "taken": 1, "copies": 9, "used": 1}


def test_one_counter_for_taken_and_used(rd):
    """What every CTA reads while one of them writes: late ones would take other pages than the table names."""
    refused(rd, taken=FAKE + 4096, used=FAKE + 4096)
    refused(rd, **{**PLACES, "taken": PLACES["used"]})


@pytest.mark.parametrize("read", ["src", "dst", "fork_lens", "free_pages", "taken"])
@pytest.mark.parametrize("written", ["lens", "copies", "used"])
def test_an_output_over_an_input(rd, written, read):
    first, last = PLACES[written], PLACES[written] + WORD * (ENTRIES[written] - 1)
    for at in (first, last, first - WORD * (ENTRIES[read] - 1)):
        refused(rd, **{**PLACES, read: at})


@pytest.mark.parametrize("one,other", [("lens", "copies"), ("lens", "used"), ("copies", "used")])
def test_an_output_over_another(rd, one, other):
    refused(rd, **{**PLACES, other: PLACES[one] + WORD * (ENTRIES[one] - 1)})
    refused(rd, **{**PLACES, one: PLACES[other] + WORD * (ENTRIES[other] - 1)})
