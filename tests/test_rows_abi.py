"""Refusals of the calls whose rows and lengths are device data, and their workspaces, on the CPU:
every call here fails its checks (or is a no-op) before any device work."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2608_10402_amd as tide
from paper_2608_10402_amd import _lib
from test_cache_abi import BAD
from test_codegen import _asm, loops_with_scratch

GOOD = _lib.make_dims(28, 4, 128, 1 / math.sqrt(128))
X = 1 << 20  # an aligned address that nothing reads: the calls fail first

CALLS = {
    "tide_page_map": dict(lens=X, want=X, n=1, bt=X, stride=4, free=X, cap=8, count=X, rows=3, lens_out=X,
                          count_out=X, row_start=X, row_task=X, row_pos=X, row_slot=X, dims=GOOD, stream=None),
    "tide_slot_append": dict(k_new=X, v_new=X, row_slot=X, rows=3, k_pool=X, v_pool=X, pages=10, bounds=X, units=X,
                             dims=GOOD, ws=X, ws_bytes=1 << 20, stream=None),
    "tide_key_bounds": dict(k_pool=X, pages=10, bt=X, stride=4, n=1, lens=X, from_lens=None, max_len=0, bounds=X,
                            units=X, dims=GOOD, ws=X, ws_bytes=1 << 20, stream=None),
    "tide_block_select": dict(q=X, row_task=X, row_pos=X, rows=3, bounds=X, units=X, pages=10, bt=X, stride=4, n=1,
                              budget=4, sink=1, recent=1, max_len=0, dims=GOOD, sel=X, ws=X, ws_bytes=1 << 20,
                              stream=None),
    "tide_sparse_attn": dict(q=X, k_pool=X, v_pool=X, pages=10, bt=X, stride=4, n=1, row_task=X, row_pos=X, rows=3,
                             sel=X, budget=4, dims=GOOD, out=X, lse=None, ws=X, ws_bytes=1 << 20, stream=None),
}


def call(name, **over):
    args = dict(CALLS[name])
    for k in over:
        assert k in args, (name, k)
    args.update(over)
    return getattr(tide.load(), name)(*(ctypes.byref(v) if isinstance(v, _lib.tide_dims) else v for v in args.values()))


POINTERS = [(n, k) for n, a in CALLS.items() for k, v in a.items() if v == X and k != "ws_bytes"]


@pytest.mark.parametrize("name,arg", POINTERS)
def test_null_pointers(name, arg):
    assert call(name, **{arg: None}) == tide.TIDE_ERR_INVALID_ARG


@pytest.mark.parametrize("name,arg", [p for p in POINTERS if p[1] in ("k_new", "v_new", "k_pool", "v_pool", "q", "out",
                                                                     "bounds", "ws")])
def test_pointers_off_16_bytes(name, arg):
    assert call(name, **{arg: X + 8}) == tide.TIDE_ERR_INVALID_ARG


@pytest.mark.parametrize("name", CALLS)
def test_shapes_and_counts(name):
    for dims, code in BAD:
        assert call(name, dims=dims) == code
    for arg in ("n", "rows"):
        if arg in CALLS[name]:
            assert call(name, **{arg: -1}) == tide.TIDE_ERR_INVALID_ARG
    main = "n" if "row_slot" not in CALLS[name] or name == "tide_page_map" else "rows"
    assert call(name, **{main: 0}) == tide.TIDE_OK
    if "pages" in CALLS[name]:
        assert call(name, pages=0) == tide.TIDE_ERR_INVALID_ARG
    if "stride" in CALLS[name]:
        assert call(name, stride=0) == tide.TIDE_ERR_INVALID_ARG
    if "ws" in CALLS[name]:
        assert call(name, ws_bytes=64) == tide.TIDE_ERR_CAPACITY


def test_rows_of_nothing():
    assert call("tide_block_select", rows=0) == tide.TIDE_OK
    assert call("tide_sparse_attn", rows=0) == tide.TIDE_OK
    assert call("tide_block_select", rows=0, budget=0) == tide.TIDE_ERR_INVALID_ARG


def test_budget_limits():
    for name in ("tide_block_select", "tide_sparse_attn"):
        assert call(name, budget=2**30 + 1) == tide.TIDE_ERR_UNSUPPORTED
    with pytest.raises(tide.TideError) as e:
        tide.tide_rows_workspace_size(tide.TIDE_OP_SPARSE_ATTN, 1, GOOD, budget=2**30 + 1)
    assert e.value.status == tide.TIDE_ERR_UNSUPPORTED
    assert tide.tide_rows_workspace_size(tide.TIDE_OP_SPARSE_ATTN, 1, GOOD, budget=2**30) > 0


def test_page_map_limits():
    assert call("tide_page_map", n=1 << 20, stride=1 << 11) == tide.TIDE_ERR_UNSUPPORTED
    assert call("tide_page_map", rows=2**31 - 1) == tide.TIDE_ERR_UNSUPPORTED
    assert call("tide_page_map", cap=-1) == tide.TIDE_ERR_INVALID_ARG


def test_bounds_and_units_go_together():
    assert call("tide_slot_append", bounds=None) == tide.TIDE_ERR_INVALID_ARG
    assert call("tide_slot_append", units=None) == tide.TIDE_ERR_INVALID_ARG
    assert call("tide_slot_append", bounds=None, units=None, ws_bytes=64) == tide.TIDE_ERR_CAPACITY


@pytest.mark.parametrize("name", ["tide_key_bounds", "tide_block_select"])
def test_max_len(name):
    assert call(name, max_len=-1) == tide.TIDE_ERR_INVALID_ARG
    assert call(name, max_len=65) == tide.TIDE_ERR_CAPACITY
    assert call(name, max_len=64, ws_bytes=64) == tide.TIDE_ERR_CAPACITY


def test_budgets():
    for over in (dict(budget=0), dict(budget=-1), dict(sink=-1), dict(recent=-1), dict(sink=3, recent=2),
                 dict(sink=2**31 - 1, recent=2**31 - 1)):
        assert call("tide_block_select", **over) == tide.TIDE_ERR_INVALID_ARG
    assert call("tide_sparse_attn", budget=0) == tide.TIDE_ERR_INVALID_ARG


def size(op, rows, dims=GOOD, **kw):
    return tide.tide_rows_workspace_size(op, rows, dims, **kw)


def test_workspace_sizes():
    assert size(tide.TIDE_OP_SLOT_APPEND, 5) == size(tide.TIDE_OP_KEY_BOUNDS, 7) == 256
    assert size(tide.TIDE_OP_BLOCK_SELECT, 3, max_len=1000) == 256 + 3 * 4 * 64 * 4   # 63 blocks: 64 scores
    assert size(tide.TIDE_OP_BLOCK_SELECT, 1 << 20, max_len=1 << 17) <= (256 << 20) + 256
    assert size(tide.TIDE_OP_BLOCK_SELECT, 1 << 20, max_len=2**31 - 1) == 256 + 4 * (1 << 27) * 4  # one row a round
    assert size(tide.TIDE_OP_BLOCK_SELECT, 0, max_len=5) == size(tide.TIDE_OP_SPARSE_ATTN, 0, budget=5) == 256
    assert size(tide.TIDE_OP_SPARSE_ATTN, 4096, budget=128) == 256
    few = size(tide.TIDE_OP_SPARSE_ATTN, 1, budget=1024)
    assert 256 < few < 1 << 20
    for op, kw in ((tide.TIDE_OP_BLOCK_SELECT, {}), (tide.TIDE_OP_SPARSE_ATTN, {}), (tide.TIDE_OP_KV_EVICT, {})):
        with pytest.raises(tide.TideError):
            size(op, 3, **kw)
    with pytest.raises(tide.TideError):
        size(tide.TIDE_OP_SLOT_APPEND, -1)


class TestBinding:
    """What the Python layer refuses by itself (host tensors; no call reaches the library)."""

    def pieces(self):
        i32 = torch.int32
        return dict(lens=torch.zeros(3, dtype=i32), want_lens=torch.zeros(3, dtype=i32),
                    block_table=torch.zeros((3, 4), dtype=i32), free_pages=torch.zeros(8, dtype=i32),
                    free_count=torch.zeros(1, dtype=i32), lens_out=torch.zeros(3, dtype=i32),
                    free_count_out=torch.zeros(1, dtype=i32), row_start=torch.zeros(4, dtype=i32),
                    row_task=torch.zeros(5, dtype=i32), row_pos=torch.zeros(5, dtype=i32),
                    row_slot=torch.zeros(5, dtype=torch.int64), dims=GOOD)

    @pytest.mark.parametrize("arg", ["want_lens", "lens_out", "free_count", "free_count_out", "row_start", "row_pos",
                                     "row_slot"])
    def test_page_map_shapes(self, arg):
        args = self.pieces()
        args[arg] = torch.zeros(args[arg].numel() + 1, dtype=args[arg].dtype)
        with pytest.raises(ValueError, match=arg):
            tide.tide_page_map(**args)

    def test_page_map_table_and_device(self):
        args = self.pieces()
        with pytest.raises(ValueError, match="block_table"):
            tide.tide_page_map(**dict(args, block_table=args["block_table"][:2]))
        with pytest.raises(ValueError, match="device"):
            tide.tide_page_map(**args)

    def test_rows_and_pools(self):
        q = torch.zeros((3, 28, 128), dtype=torch.bfloat16)
        pool = torch.zeros((5, 4, 16, 128), dtype=torch.bfloat16)
        bt = torch.zeros((2, 6), dtype=torch.int32)
        row = torch.zeros(3, dtype=torch.int32)
        sel = torch.zeros((3, 4, 8), dtype=torch.int32)
        bounds, units = torch.zeros((5, 4, 2, 128), dtype=torch.int8), torch.zeros((5, 4), dtype=torch.int8)
        with pytest.raises(ValueError, match="sel"):
            tide.tide_block_select(q, row, row, bounds, units, bt, 9, GOOD, sel)
        with pytest.raises(ValueError, match="sel"):
            tide.tide_sparse_attn(q, pool, pool, bt, row, row, sel[:, :3], GOOD, q)
        with pytest.raises(ValueError, match="row_pos"):
            tide.tide_sparse_attn(q, pool, pool, bt, row, row[:2], sel, GOOD, q)
        with pytest.raises(ValueError, match="q must"):
            tide.tide_block_select(q[:2], row, row, bounds, units, bt, 8, GOOD, sel)
        with pytest.raises(ValueError, match="units"):
            tide.tide_block_select(q, row, row, bounds, units[:, :3], bt, 8, GOOD, sel)
        with pytest.raises(ValueError, match="lse"):
            tide.tide_sparse_attn(q, pool, pool, bt, row, row, sel, GOOD, q, torch.zeros(3, 27))
        k = torch.zeros((3, 4, 128), dtype=torch.bfloat16)
        with pytest.raises(ValueError, match="together"):
            tide.tide_slot_append(k, k, torch.zeros(3, dtype=torch.int64), pool, pool, GOOD, bounds)
        with pytest.raises(ValueError, match="k_new"):
            tide.tide_slot_append(k[:2], k, torch.zeros(3, dtype=torch.int64), pool, pool, GOOD)
        with pytest.raises(ValueError, match="bounds"):
            tide.tide_key_bounds(pool, bt, row[:2], bounds[:4], units, GOOD)
        with pytest.raises(ValueError, match="device"):
            tide.tide_sparse_attn(q, pool, pool, bt, row, row, sel, GOOD, q)

    def test_page_table_starts_empty(self):
        t = tide.PageTable(3, 4, 7, device="cpu")
        assert t.free_pages.tolist() == [6, 5, 4, 3, 2, 1, 0] and t.free_count.tolist() == [7]
        assert t.lens.tolist() == [0, 0, 0] and tuple(t.block_table.shape) == (3, 4)
        assert tide.PageTable(3, 4, [9, 2], device="cpu").free_pages.tolist() == [9, 2]
        task, pos, slot = t.new_rows(2)
        assert task.tolist() == pos.tolist() == slot.tolist() == [-1, -1] and slot.dtype == torch.int64

    def test_new_bounds(self):
        kv = tide.PagedKV(3, 8, 2, 64, [[0, 1, 2]], device="cpu")
        b, u = kv.new_bounds()
        assert tuple(b.shape) == (3, 2, 2, 64) and tuple(u.shape) == (3, 2) and b.dtype == u.dtype == torch.int8


@pytest.mark.parametrize("src", ["page_map.hip", "key_bounds.hip", "block_select.hip", "sparse_attn.hip", "sparse_shared.hip"])
def test_no_scratch_access_inside_loops(tmp_path, src):
    found = loops_with_scratch(_asm(tmp_path, src))
    assert found or src == "key_bounds.hip"
    bad = [x for x in found if x[2]]
    assert not bad, bad
