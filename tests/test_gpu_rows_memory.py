"""Memory of the calls whose rows and lengths are device data (needs an MI355X): which of a page map's arrays may be the
same, workspaces that graphs use, and the bounds of pages that were cut."""
import numpy as np
import pytest
import torch

import paper_2608_10402_amd as tide
import rows_reference as W
from test_gpu_rows import D, HKV, HQ, Sparse, dev, engine, host, rows_to_dev

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


def test_a_graph_keeps_its_workspace():
    """A captured choice and attention of 64 rows, replayed after eager calls of fewer rows, whose split lists need
    more memory, and of more: the results of the eager call each time, and nothing written to other tensors."""
    s = Sparse(41, [4096, 4000], 28, 4, 128)
    q, task, pos = s.rows(64)
    q, task, pos = rows_to_dev(q), dev(task), dev(pos)
    kv, bounds = s.p.kv, s.p.kv.new_bounds()
    kv.key_bounds(dev(s.lens), bounds)

    def call(n):
        sel = kv.select_blocks(q[:n], task[:n], pos[:n], bounds, 128, 1, 2, out=torch.full((n, 4, 128), -1, device="cuda",
                                                                                          dtype=torch.int32))
        return sel, kv.sparse(q[:n], task[:n], pos[:n], sel)

    want = call(64)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = call(64)
    few = call(32)
    more = torch.cat([q] * 40), torch.cat([task] * 40), torch.cat([pos] * 40)
    for i in range(3):
        filler = [torch.full((1 << k,), 7, dtype=torch.uint8, device="cuda") for k in range(8, 25)]
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
        assert all((x == 7).all() for x in filler), i
        for x in got:
            x.fill_(3)
        assert all(torch.equal(a, b) for a, b in zip(call(32), few)), i
        kv.select_blocks(*more, bounds, 128, 1, 2)
        torch.zeros(1000, device="cuda").sum().item()


@pytest.mark.parametrize("by", ["key_bounds", "append"])
def test_bounds_of_a_page_that_was_cut(by):
    """A context that ends inside a page leaves the page the bounds of what it held, here of a key that is not a
    number and of a large one; from_lens = lens - 1 brings the last pages up to date, as the next append does."""
    rng = np.random.default_rng(42)
    kv, table, bounds = engine(3, 20, 60)
    lens, cut = [200, 110, 96], [165, 83, 96]  # inside pages 10 and 5; the third stays
    rows = table.new_rows(sum(lens))
    table.map(dev(lens), rows)
    k = rng.standard_normal((sum(lens), HKV, D))
    k[180:200], k[200 + 90] = 1e6, np.nan  # positions 180 .. of the first task, 90 of the second
    k = rows_to_dev(k)
    kv.append_slots(k, k, rows[2], bounds)
    before = [x.cpu().numpy() for x in bounds]
    table.map(dev(cut), table.new_rows(0))
    q = rows_to_dev(rng.standard_normal((3, HQ, D)))
    task, pos = dev([0, 1, 2]), dev([x - 1 for x in cut])

    # what the cut leaves: the bounds as they were, which a choice goes by
    bt, g = table.block_table.cpu().numpy(), HQ // HKV
    assert (before[1][bt[1, 5]] == W.NONE).all()
    assert (kv.select_blocks(q, task, pos, bounds, 2)[1] == 5).any(-1).all()

    held, last = host(kv.k_pool), list(cut)
    if by == "key_bounds":
        kv.key_bounds(table.lens, bounds, from_lens=table.lens - 1)
    else:
        rows, one = table.new_rows(3), rows_to_dev(rng.standard_normal((3, HKV, D)))
        last = [x + 1 for x in cut]
        table.map(dev(last), rows)
        kv.append_slots(one, one, rows[2], bounds)
        bt, held, pos = table.block_table.cpu().numpy(), host(kv.k_pool), dev([x - 1 for x in last])
    after = [x.cpu().numpy() for x in bounds]
    changed = {int(bt[b, (n - 1) // 16]) for b, n in enumerate(last)}
    for page in range(60):
        if page not in changed:
            assert np.array_equal(after[0][page], before[0][page]) and np.array_equal(after[1][page], before[1][page])
    for b, n in enumerate(last):
        page = bt[b, (n - 1) // 16]
        for h in range(HKV):
            hi, lo, s = W.bounds_of(held[page, h, : (n - 1) % 16 + 1])
            assert after[1][page, h] == s and np.array_equal(after[0][page, h], np.stack((hi, lo)))
    sel, hq = kv.select_blocks(q, task, pos, bounds, 4, 1, 0).cpu().numpy(), host(q)
    for b, n in enumerate(last):
        at = bt[b, : W.pages_of(n)]
        for h in range(HKV):
            s = W.scores(hq[b, h * g:(h + 1) * g], after[0][at, h, 0], after[0][at, h, 1], after[1][at, h])
            assert sel[b, h].tolist() == W.choose(s, len(at), 4, 1, 0)
