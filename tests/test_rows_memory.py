"""Memory of the calls whose rows and lengths are device data, on the CPU: arrays that overlap are refused."""
import pytest

import paper_2608_10402_amd as tide
from test_rows_abi import call

N, STRIDE, CAP, ROWS = 5, 7, 11, 13
SPAN = 1 << 24  # between addresses that nothing reads: the calls fail first
INPUTS = {"lens": 4 * N, "want": 4 * N, "count": 4}
WRITTEN = {"bt": 4 * N * STRIDE, "free": 4 * CAP, "lens_out": 4 * N, "count_out": 4, "row_start": 4 * (N + 1),
           "row_task": 4 * ROWS, "row_pos": 4 * ROWS, "row_slot": 8 * ROWS}
BYTES = dict(INPUTS, **WRITTEN)


def page_map(**over):
    args = {name: SPAN * (i + 1) for i, name in enumerate(BYTES)}
    return call("tide_page_map", **dict(args, n=N, stride=STRIDE, cap=CAP, rows=ROWS, **over))


def address(name):
    return SPAN * (list(BYTES).index(name) + 1)


@pytest.mark.parametrize("written", WRITTEN)
@pytest.mark.parametrize("other", BYTES)
def test_page_map_refuses_arrays_that_overlap(written, other):
    """What is written and any other array: from the same address on (lens_out and lens, count_out and count may
    be the same), and by the last or the first 4 bytes."""
    if written == other:
        return
    at, size, mine = address(other), BYTES[other], BYTES[written]
    if (written, other) not in (("lens_out", "lens"), ("count_out", "count")):
        assert page_map(**{written: at}) == tide.TIDE_ERR_INVALID_ARG
    if size > 4:
        assert page_map(**{written: at + size - 4}) == tide.TIDE_ERR_INVALID_ARG
    if mine > 4:
        assert page_map(**{written: at - mine + 4}) == tide.TIDE_ERR_INVALID_ARG


def test_page_map_refuses_wanted_lengths_in_the_place_of_the_new_ones():
    """A refused task's length would take the place of the one it is compared with."""
    assert page_map(lens_out=address("want")) == tide.TIDE_ERR_INVALID_ARG
    assert page_map(want=address("lens") + 4, lens_out=address("lens")) == tide.TIDE_ERR_INVALID_ARG
