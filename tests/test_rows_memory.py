"""Memory of the calls whose rows and lengths are device data, on the CPU: arrays that overlap are refused, and
workspaces hold what smaller calls need and live as long as graphs may use them."""
import ctypes
import math
import weakref

import pytest
import torch

import paper_2608_10402_amd as tide
from paper_2608_10402_amd import _lib, kvcache
from test_cache_abi import BAD
from test_rows_abi import GOOD, call

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


# ---- workspaces ----------------------------------------------------------------------------------------

HEADS = [(28, 4, 128), (32, 8, 128), (8, 8, 64), (1, 1, 64), (16, 1, 128), (512, 512, 64)]
ROWS_UP = [0, 1, 2, 3, 8, 31, 32, 33, 63, 64, 65, 255, 256, 257, 300, 4096, 1 << 20, 2**31 - 1]
BUDGETS_UP = [1, 2, 94, 95, 96, 127, 128, 129, 512, 520, 1024, 1 << 15, 1 << 30]
LENGTHS_UP = [1, 16, 1000, 1024, 1025, 4096, 1 << 17, 9 << 20, (9 << 20) + 1, 1 << 24, (1 << 24) + 1, 2**31 - 1]


def size(op, rows, dims, n):
    return tide.tide_rows_workspace_size(op, rows, dims, budget=n, max_len=n)


def bound(op, rows, dims, n):
    return tide.tide_rows_workspace_bound(op, rows, dims, budget=n, max_len=n)


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("op,up", [(tide.TIDE_OP_BLOCK_SELECT, LENGTHS_UP), (tide.TIDE_OP_SPARSE_ATTN, BUDGETS_UP),
                                   (tide.TIDE_OP_SLOT_APPEND, [1]), (tide.TIDE_OP_KEY_BOUNDS, [1])])
def test_workspace_bounds_hold_every_smaller_call(op, up, heads):
    """Sizes fall where more rows are no longer split and where rounds leave a rest; bounds never do."""
    dims = _lib.make_dims(*heads, 1 / math.sqrt(heads[2]))
    sizes = [[size(op, r, dims, n) for n in up] for r in ROWS_UP]
    bounds = [[bound(op, r, dims, n) for n in up] for r in ROWS_UP]
    for i in range(len(ROWS_UP)):
        for j in range(len(up)):
            assert bounds[i][j] >= max(max(x[: j + 1]) for x in sizes[: i + 1]), (ROWS_UP[i], up[j])
            assert i == 0 or bounds[i][j] >= bounds[i - 1][j]
            assert j == 0 or bounds[i][j] >= bounds[i][j - 1]


def test_workspace_bounds_are_close():
    """A bound is at most what the largest smaller call takes, or the limit of a round of scores."""
    sparse = [size(tide.TIDE_OP_SPARSE_ATTN, r, GOOD, 128) for r in range(1, 65)]
    assert size(tide.TIDE_OP_SPARSE_ATTN, 64, GOOD, 128) < max(sparse)  # sizes do fall
    assert bound(tide.TIDE_OP_SPARSE_ATTN, 64, GOOD, 128) == bound(tide.TIDE_OP_SPARSE_ATTN, 4096, GOOD, 128) == max(sparse)
    assert bound(tide.TIDE_OP_SPARSE_ATTN, 4096, GOOD, 90) == 256
    assert bound(tide.TIDE_OP_BLOCK_SELECT, 300, GOOD, 1 << 24) == 256 + (256 << 20)
    assert bound(tide.TIDE_OP_BLOCK_SELECT, 3, GOOD, 1000) == size(tide.TIDE_OP_BLOCK_SELECT, 3, GOOD, 1000)
    assert bound(tide.TIDE_OP_BLOCK_SELECT, 3, GOOD, 2**31 - 1) == size(tide.TIDE_OP_BLOCK_SELECT, 3, GOOD, 2**31 - 1)


def test_workspace_bounds_refuse_what_sizes_refuse():
    out, fn = ctypes.c_size_t(0), tide.load().tide_rows_workspace_bound
    for dims, code in BAD:
        assert fn(tide.TIDE_OP_KEY_BOUNDS, 1, 1, 1, None if dims is None else ctypes.byref(dims), ctypes.byref(out)) == code
    assert fn(tide.TIDE_OP_KEY_BOUNDS, 1, 1, 1, ctypes.byref(GOOD), None) == tide.TIDE_ERR_INVALID_ARG
    for op, rows, n, code in ((tide.TIDE_OP_KV_EVICT, 3, 1, tide.TIDE_ERR_INVALID_ARG),
                              (tide.TIDE_OP_SLOT_APPEND, -1, 1, tide.TIDE_ERR_INVALID_ARG),
                              (tide.TIDE_OP_BLOCK_SELECT, 3, 0, tide.TIDE_ERR_INVALID_ARG),
                              (tide.TIDE_OP_SPARSE_ATTN, 3, 0, tide.TIDE_ERR_INVALID_ARG),
                              (tide.TIDE_OP_SPARSE_ATTN, 3, 2**30 + 1, tide.TIDE_ERR_UNSUPPORTED)):
        with pytest.raises(tide.TideError) as e:
            bound(op, rows, GOOD, n)
        assert e.value.status == code


class Engine:
    """A PagedKV on the host whose entry points only check and note the workspaces that they get."""

    def __init__(self, monkeypatch):
        self.used = []
        self.kv = tide.PagedKV(3, 28, 4, 128, torch.zeros((2, 1 << 14), dtype=torch.int32), device="cpu")
        ops = dict(tide_slot_append=tide.TIDE_OP_SLOT_APPEND, tide_key_bounds=tide.TIDE_OP_KEY_BOUNDS,
                   tide_block_select=tide.TIDE_OP_BLOCK_SELECT, tide_sparse_attn=tide.TIDE_OP_SPARSE_ATTN)
        for name, op in ops.items():
            monkeypatch.setattr(kvcache._lib, name, lambda *a, op=op: self.note(op, *a))

    def note(self, op, *args):
        ws = [x for x in args if isinstance(x, torch.Tensor) and x.dtype == torch.uint8][-1]
        need = 256
        if op == tide.TIDE_OP_BLOCK_SELECT:
            need = size(op, args[1].shape[0], GOOD, args[11] or self.kv.block_table.shape[1] * 16)
        if op == tide.TIDE_OP_SPARSE_ATTN:
            need = size(op, args[4].shape[0], GOOD, args[6].shape[2])
        if ws.numel() < need:
            raise tide.TideError(tide.TIDE_ERR_CAPACITY, "too small")
        self.used.append(ws)

    def rows(self, n):
        return (torch.zeros((n, 28, 128), dtype=torch.bfloat16), torch.zeros(n, dtype=torch.int32),
                torch.zeros(n, dtype=torch.int32))

    def sparse(self, n, budget):
        self.kv.sparse(*self.rows(n), torch.zeros((n, 4, budget), dtype=torch.int32))
        return self.used[-1]

    def select(self, n, max_len=0):
        self.kv.select_blocks(*self.rows(n), self.kv.new_bounds(), 8, max_len=max_len)
        return self.used[-1]

    def append(self):
        k = torch.zeros((2, 4, 128), dtype=torch.bfloat16)
        self.kv.append_slots(k, k, torch.zeros(2, dtype=torch.int64), self.kv.new_bounds())
        return self.used[-1]


def test_a_smaller_call_keeps_the_workspace(monkeypatch):
    """What a captured graph of the larger call uses: fewer rows need more, since their lists are split."""
    for first in ("append", "sparse"):
        e = Engine(monkeypatch)
        if first == "append":
            e.append()
        at = e.sparse(64, 128).data_ptr()
        for n in (64, 63, 32, 7, 1):
            for budget in (128, 100, 3):
                assert e.sparse(n, budget).data_ptr() == at, (n, budget)
        assert e.append().data_ptr() == at


def test_a_shorter_choice_keeps_the_workspace(monkeypatch):
    e = Engine(monkeypatch)
    at = e.select(300, 1 << 18).data_ptr()
    for n, most in ((300, (1 << 18) - 5), (299, 1 << 18), (17, 4096), (1, 1)):
        assert e.select(n, most).data_ptr() == at
    assert e.append().data_ptr() == at


def test_replaced_workspaces_live_on(monkeypatch):
    """A graph that was captured with one writes to it at each replay, whatever larger calls came since; together
    the replaced ones take less than the present one."""
    e = Engine(monkeypatch)
    alive = [weakref.ref(e.append())]
    for n in (1, 8, 30, 300, 900, 3000):
        e.sparse(n, 1000)
        alive.append(weakref.ref(e.select(n)))
    e.used.clear()
    each = {x().data_ptr(): x().numel() for x in alive}  # (all are there)
    assert len(each) > 2 and sum(each.values()) < 2 * max(each.values())


def test_other_calls_do_not_replace_it(monkeypatch):
    e = Engine(monkeypatch)
    at = e.sparse(64, 128).data_ptr()
    e.kv.workspace(1 << 24)  # as a decode of long contexts does
    assert e.sparse(64, 128).data_ptr() == at and e.select(1, 16).data_ptr() == at


def test_a_choice_past_the_table_takes_no_memory(monkeypatch):
    """max_len above what the table holds is refused by the call, which is made with the table's workspace."""
    e = Engine(monkeypatch)
    with pytest.raises(tide.TideError):
        e.select(1, 2**31 - 1)
    assert e.append().numel() < 1 << 22


@pytest.mark.parametrize("out", [1 << 24, (1 << 24) + 3 * 28 * 128 * 2 - 16, (1 << 24) - 3 * 28 * 128 * 2 + 16])
def test_attention_over_lists_refuses_outputs_over_queries(out):
    """Rows that are taken again read their queries after outputs were written."""
    assert call("tide_sparse_attn", q=1 << 24, out=out) == tide.TIDE_ERR_INVALID_ARG
