"""Memory of the calls whose rows and lengths are device data (needs an MI355X): which of a page map's arrays may be the
same."""
import numpy as np
import pytest
import torch

import paper_2608_10402_amd as tide
import rows_reference as W
from test_gpu_rows import dev, engine

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [40, 5000])  # with the rows by the same kernel, and by one of their own
def test_page_map_to_its_own_lengths(rows):
    """The cached lengths as the wanted ones: nothing moves, all rows are padding."""
    kv, table, bounds = engine(3, 20, 40)
    table.map(dev([30, 0, 100]), table.new_rows(rows))
    before = [x.clone() for x in (table.block_table, table.lens, table.free_pages, table.free_count)]
    got = [torch.full_like(x, 5) for x in table.new_rows(rows)]
    table.map(table.lens, got)
    for x, y in zip((table.block_table, table.lens, table.free_pages, table.free_count), before):
        assert torch.equal(x, y)
    assert all((x == -1).all() for x in got) and table.row_start.tolist() == [0] * 4


@pytest.mark.parametrize("rows", [40, 5000])
def test_page_map_refuses_to_replace_the_wanted_lengths(rows):
    """Two tasks want more pages (or rows) than there are: with their wanted lengths replaced by the granted ones, which the
    rows' kernel compares them with, the refused task's rows would lie in pages of others."""
    kv, table, bounds = engine(2, 300, 4)
    want = dev([60, 2000])
    out = table.new_rows(rows)
    args = dict(lens=table.lens, want_lens=want, block_table=table.block_table, free_pages=table.free_pages,
                free_count=table.free_count, free_count_out=table.free_count, row_start=table.row_start,
                row_task=out[0], row_pos=out[1], row_slot=out[2], dims=tide.make_dims(1, 1, 64, 1.0))
    for lens_out in (want, want.view(2), table.row_start[:2], out[0][:2], table.block_table.view(-1)[:2]):
        with pytest.raises(tide.TideError) as e:
            tide.tide_page_map(lens_out=lens_out, **args)
        assert e.value.status == tide.TIDE_ERR_INVALID_ARG
    assert want.tolist() == [60, 2000] and table.lens.tolist() == [0, 0] and (out[0] == -1).all()
    tide.tide_page_map(lens_out=table.lens, **args)
    lens, _, _, _, _, expect = W.page_map([0, 0], [60, 2000], np.zeros((2, 300)), [3, 2, 1, 0], 4, rows)
    assert lens == ([60, 0] if rows >= 60 else [0, 0]) and table.lens.tolist() == lens
    assert np.array_equal(np.stack([x.cpu().numpy() for x in out], 1), expect)
