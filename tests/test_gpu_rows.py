"""Page maps, appends by slots, key bounds, the choice of blocks and attention over them on the GPU,
against tests/rows_reference.py: whole numbers equal, outputs within bounds derived from the roundings."""
import numpy as np
import pytest
import torch

import cache_reference as R
import paper_2608_10402_amd as tide
import rows_reference as W

pytestmark = pytest.mark.gpu

PAGE = 16


def dev(x, dtype=np.int32):
    return torch.from_numpy(np.array(x, dtype)).cuda()


def rows_to_dev(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(torch.bfloat16).cuda()


def host(t):
    return t.double().cpu().numpy()


# ---- page maps --------------------------------------------------------------------------------------

def run_map(lens, want, table, free, count, num_rows, in_place=False):
    n = len(lens)
    d = dict(lens=dev(lens), want_lens=dev(want), block_table=dev(table), free_pages=dev(free),
             free_count=dev([count]), row_start=dev(np.zeros(n + 1)), row_task=dev(np.zeros(num_rows)),
             row_pos=dev(np.zeros(num_rows)), row_slot=dev(np.zeros(num_rows), np.int64))
    d["lens_out"] = d["lens"] if in_place else dev(np.full(n, -7))
    d["free_count_out"] = d["free_count"] if in_place else dev([-7])
    tide.tide_page_map(dims=tide.make_dims(1, 1, 64, 1.0), **d)
    rows = np.stack([d[x].cpu().numpy().astype(np.int64) for x in ("row_task", "row_pos", "row_slot")], 1)
    return tuple(d[x].cpu().numpy() for x in ("lens_out", "block_table", "free_pages")) + (
        int(d["free_count_out"]), d["row_start"].cpu().numpy(), rows)


def same_map(*args, **kw):
    got, want = run_map(*args, **kw), W.page_map(*args)
    for g, w, name in zip(got, want, ("lens", "table", "free pages", "count", "row start", "rows")):
        assert np.array_equal(g, w), name
    return got


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 175, 1023, 1024, 1025, 5000])
@pytest.mark.parametrize("most", [1, 40])
def test_page_map(n, most):
    """Growing, shrinking and idle tasks, in a pool that is large enough, too small, and with too few rows."""
    rng = np.random.default_rng(n + most)
    stride = 12
    lens = rng.integers(0, 150, n)
    move = rng.integers(-most, most + 1, n) if most > 1 else np.ones(n, int)
    want = np.clip(lens + move, 0, stride * PAGE)
    held = sum(W.pages_of(x) for x in lens)
    ids = rng.permutation(held + 4 * n + 3)
    table, at = np.full((n, stride), -5), 0
    for b in range(n):
        m = W.pages_of(lens[b])
        table[b, :m] = ids[at:at + m]
        at += m
    total = int(np.maximum(0, want - lens).sum())
    free = np.full(ids.size, -9)
    for count, rows in ((4 * n + 3, total), (4 * n + 3, total + 70), (n // 40, total), (4 * n + 3, total * 2 // 3),
                        (0, 0), (4 * n + 3, total + 5000)):
        free[:count] = ids[at:at + count]
        same_map(lens, want, table, free, count, rows)
        same_map(lens, want, table, free, count, rows, in_place=True)


def test_page_map_of_lengths_that_are_none():
    big = 2**31 - 1
    same_map([5, -1, 7, 200, 8, 40], [-3, 9, big, 3, 65, 64], np.arange(24).reshape(6, 4), np.arange(50, 60), 10, 40)
    same_map([0, 0, 0], [big, big, 64], np.zeros((3, 4), int), np.arange(9), 9, 100)


def test_page_map_of_long_tasks():
    """Requests whose sums pass 32 bits are refused, and a long task's pages and rows are many a thread."""
    n, stride = 40, 6000
    lens = np.arange(n) * 3
    want = np.full(n, stride * PAGE)
    want[7] = 5
    same_map(lens, want, np.zeros((n, stride), int), np.arange(20000), 20000, 150000)
    same_map(want, lens, np.arange(n * stride).reshape(n, stride), np.zeros(n * stride, int), 0, 50)


@pytest.mark.parametrize("n,pages,room", [(3, 190000, 10**6), (2500, 260, 10**6), (2100, 300, 50000), (1, 600000, 10**6)])
def test_page_map_of_large_tables(n, pages, room):
    """Tables whose returned pages are moved by workgroups of their own, some past the stack's end; in place too."""
    rng = np.random.default_rng(n)
    lens = rng.integers(0, PAGE * pages + 1, n)
    want = np.where(rng.random(n) < 0.6, rng.integers(0, lens + 1), np.minimum(lens + rng.integers(0, 40, n), PAGE * pages))
    want[0], lens[-1] = 0, PAGE * pages
    table = rng.integers(0, 2**31 - 1, (n, pages))
    free = rng.integers(0, 2**31 - 1, min(room, 10 + W.pages_of(lens.max()) * n))
    for in_place in (False, True):
        same_map(lens, want, table, free, 10, 3000, in_place=in_place)


def test_page_map_keeps_the_stack_in_its_array():
    """Pages that do not fit are dropped; a count out of range is taken as the nearest that is not."""
    table = np.arange(30).reshape(3, 10)
    same_map([160, 100, 0], [10, 0, 20], table, np.full(6, 77), 2, 30)
    same_map([160, 100, 0], [160, 101, 20], table, np.full(6, 77), 9, 30)
    same_map([160, 100, 0], [160, 101, 20], table, np.full(6, 77), -4, 30)
    same_map([160, 100, 5], [160, 100, 5], table, np.zeros(0, int), 0, 0)


def test_page_map_of_bad_free_pages():
    got = same_map([0, 16], [20, 17], np.zeros((2, 4), int), [-3, 5, -8], 3, 40)
    assert (got[5][:16, 2] == -1).all() and got[5][16, 2] == 5 * PAGE


# ---- appends and bounds -------------------------------------------------------------------------------

def make_table(rng, lens, extra=3):
    n = [W.pages_of(x) for x in lens]
    pages = sum(n) + extra
    order = rng.permutation(pages)
    table = np.full((len(lens), max(max(n), 1)), pages + 7)  # past a context: never read
    at = 0
    for b, k in enumerate(n):
        table[b, :k] = order[at:at + k]
        at += k
    return table.astype(np.int32), pages


class Pools:
    def __init__(self, rng, pages, hq, hkv, d, table, scale=1.0):
        self.kv = tide.PagedKV(pages, hq, hkv, d, table, fill_canary=False)
        self.k, self.v = (R.bf16(rng.standard_normal((pages, hkv, PAGE, d)) * scale) for _ in range(2))
        self.kv.k_pool.copy_(rows_to_dev(self.k))
        self.kv.v_pool.copy_(rows_to_dev(self.v))
        self.bounds = self.kv.new_bounds()
        self.b0 = rng.integers(-128, 128, tuple(self.bounds[0].shape)).astype(np.int8)
        self.u0 = rng.integers(-128, 128, tuple(self.bounds[1].shape)).astype(np.int8)
        self.bounds[0].copy_(torch.from_numpy(self.b0))
        self.bounds[1].copy_(torch.from_numpy(self.u0))

    def expect(self, page, n):
        """The bounds of the first n slots of a page go into the copies."""
        for h in range(self.k.shape[1]):
            hi, lo, s = W.bounds_of(self.k[page, h, :n])
            self.b0[page, h], self.u0[page, h] = np.stack((hi, lo)), s

    def check(self):
        assert np.array_equal(host(self.kv.k_pool), self.k, equal_nan=True)
        assert np.array_equal(host(self.kv.v_pool), self.v, equal_nan=True)
        assert np.array_equal(self.bounds[1].cpu().numpy(), self.u0)
        assert np.array_equal(self.bounds[0].cpu().numpy(), self.b0)


def rows_of(prefix, extend):
    task = np.repeat(np.arange(len(prefix)), extend)
    return task, np.concatenate([np.arange(p, p + e) for p, e in zip(prefix, extend)])


APPEND = [  # prefix, extend, kv heads, d
    ([0], [1], 1, 64), ([15], [1], 2, 128), ([3, 0, 40], [5, 33, 0], 4, 128), ([7, 16, 31], [60, 16, 2], 5, 64),
    ([1000], [129], 3, 128), ([0] * 40, [17] * 40, 1, 128), (list(range(33)), [1] * 33, 8, 128), ([14], [4], 64, 64),
    # more rows x kv heads than are taken one by one: windows of rows, few and many first rows of pages in each
    ([5, 100], [210, 61], 64, 64), (list(range(70, 370)), [1] * 300, 64, 64), ([3] * 37, [7] * 37, 65, 128),
    # and longer windows
    ([5, 100], [700, 401], 64, 64), ([i % 17 for i in range(340)], [1 + i % 5 for i in range(340)], 65, 64)]


@pytest.mark.parametrize("prefix,extend,hkv,d", APPEND)
@pytest.mark.parametrize("with_bounds", [True, False])
def test_append_by_slots(prefix, extend, hkv, d, with_bounds):
    """The rows' slots, the bounds of their pages, and nothing else; padding rows between."""
    rng = np.random.default_rng(len(prefix) + d)
    table, pages = make_table(rng, np.array(prefix) + extend)
    p = Pools(rng, pages, hkv, hkv, d, table)
    task, pos = rows_of(prefix, extend)
    k, v = (R.bf16(rng.standard_normal((task.size, hkv, d)) * 2.0 ** rng.integers(-9, 9, (task.size, hkv, 1)))
            for _ in range(2))
    page, slot = table[task, pos // PAGE].astype(np.int64), pos % PAGE
    at = page * PAGE + slot
    put = np.where(rng.random(task.size + 3) < 0.5, -1, -2**40)  # padding before and behind
    put[1:1 + task.size] = at
    pad = [((1, 2), (0, 0), (0, 0))]
    p.kv.append_slots(rows_to_dev(np.pad(k, *pad)), rows_to_dev(np.pad(v, *pad)), dev(put, np.int64),
                      p.bounds if with_bounds else None)
    p.k[page, :, slot], p.v[page, :, slot] = k, v
    if with_bounds:
        for x in set(page):
            p.expect(x, slot[page == x].max() + 1)
    p.check()


def test_append_of_slots_past_the_pool(monkeypatch):
    rng = np.random.default_rng(1)
    p = Pools(rng, 3, 8, 2, 64, [[0, 1, 2]])
    k = R.bf16(rng.standard_normal((4, 2, 64)))
    slots = [48, 20, 2**40, -1]
    p.kv.append_slots(rows_to_dev(k), rows_to_dev(k), dev(slots, np.int64), p.bounds)
    p.k[1, :, 4] = p.v[1, :, 4] = k[1]
    p.expect(1, 5)
    p.check()
    monkeypatch.setenv("TIDE_DEBUG_CHECKS", "1")
    with pytest.raises(tide.TideError) as e:
        p.kv.append_slots(rows_to_dev(k), rows_to_dev(k), dev(slots, np.int64), p.bounds)
    assert e.value.status == tide.TIDE_ERR_PAGE_RANGE
    p.kv.append_slots(rows_to_dev(k), rows_to_dev(k), dev([-1, 20, -5, -1], np.int64), p.bounds)
    p.check()


@pytest.mark.parametrize("d", [64, 128])
def test_bounds_at_the_edges_of_the_format(d):
    """Zeros of both signs, subnormals, the least and largest values, NaN and infinities: one page each."""
    top = float.fromhex("0x1.fep127")
    values = [0.0, -0.0, 2.0 ** -133, -(2.0 ** -133), top, -top, float.fromhex("0x1.fcp127"), np.nan, np.inf, -np.inf,
              127 * 2.0 ** -120, 127.5 * 2.0 ** -120, 126.5 * 2.0 ** -120, 1.984375, 1.9921875, -1.0, 2.0 ** -113]
    k = np.zeros((len(values), 1, PAGE, d))
    for i, x in enumerate(values):
        k[i, 0, i % PAGE, (7 * i) % d] = x
        k[i, 0, (i + 3) % PAGE, (7 * i + 1) % d] = -2.0 ** -133
        k[i, 0, (i + 5) % PAGE, (7 * i + 2) % d] = 2.0 ** -133
    rng = np.random.default_rng(1)
    p = Pools(rng, len(values), 1, 1, d, [list(range(len(values)))])
    p.k = R.bf16(k)
    assert np.array_equal(p.k, k, equal_nan=True)
    p.kv.k_pool.copy_(rows_to_dev(k))
    p.kv.key_bounds(dev([len(values) * PAGE]), p.bounds)
    for i in range(len(values)):
        p.expect(i, PAGE)
    p.check()


@pytest.mark.parametrize("lens,start,hkv,d", [
    ([1], None, 1, 64), ([16, 17, 0, 255], None, 2, 128), ([300, 1000, 5], [16, 999, 5], 5, 64),
    ([100, 64, 200], [0, 47, -3], 8, 128), ([40] * 60, list(range(60)), 4, 128)])
@pytest.mark.parametrize("max_len", [0, 130])
def test_key_bounds(lens, start, hkv, d, max_len):
    rng = np.random.default_rng(len(lens) + d)
    table, pages = make_table(rng, lens)
    if max_len > table.shape[1] * PAGE:
        max_len = table.shape[1] * PAGE
    p = Pools(rng, pages, hkv, hkv, d, table, scale=4.0)
    p.kv.key_bounds(dev(lens), p.bounds, None if start is None else dev(start), max_len)
    for b, n in enumerate(lens):
        n = min(n, max_len) if max_len else n
        for i in range(max(0, start[b] if start else 0) // PAGE, W.pages_of(n)):
            if (start[b] if start else 0) < n:
                p.expect(table[b, i], min(PAGE, n - PAGE * i))
    p.check()


def test_key_bounds_of_bad_pages_and_lengths(monkeypatch):
    """Page ids out of range are skipped; lengths past the table stop at its end, negative ones are none."""
    rng = np.random.default_rng(9)
    table = np.array([[0, -1, 2], [3, 2**31 - 1, 5], [1, 1, 1]], np.int32)
    p = Pools(rng, 6, 2, 2, 64, table)
    lens = [48, 2**31 - 1, -5]
    p.kv.key_bounds(dev(lens), p.bounds)
    for x in (0, 2, 3, 5):
        p.expect(x, PAGE)
    p.check()
    monkeypatch.setenv("TIDE_DEBUG_CHECKS", "1")
    with pytest.raises(tide.TideError) as e:
        p.kv.key_bounds(dev(lens), p.bounds)
    assert e.value.status == tide.TIDE_ERR_PAGE_RANGE


# ---- the choice of blocks -------------------------------------------------------------------------------

class Choice:
    """Tasks of `lens` positions whose pages have random bounds."""

    def __init__(self, seed, lens, hq, hkv, d, pool=None, levels=127):
        self.rng = rng = np.random.default_rng(seed)
        self.lens, self.hq, self.hkv, self.d = lens, hq, hkv, d
        self.table, pages = make_table(rng, lens)
        if pool is not None:  # few pages, listed many times
            pages = pool
            self.table = rng.integers(0, pool, self.table.shape).astype(np.int32)
        lo = rng.integers(-levels, levels + 1, (pages, hkv, 1, d))
        hi = np.minimum(127, lo + rng.integers(0, levels + 1, lo.shape))
        self.bounds = np.concatenate((hi, lo), 2).astype(np.int8)
        self.units = rng.integers(-9, -4, (pages, hkv)).astype(np.int8)
        self.kv = tide.PagedKV(1, hq, hkv, d, self.table, fill_canary=False)

    def queries(self, n):
        return R.bf16(self.rng.standard_normal((n, self.hq, self.d)) * 2.0 ** self.rng.integers(-3, 4, (n, self.hq, 1)))

    def expect(self, q, task, pos, budget, sink, recent):
        g = self.hq // self.hkv
        out = np.full((len(task), self.hkv, budget), -77)
        for r, (b, p) in enumerate(zip(task, pos)):
            if b < 0 or p < 0:
                continue
            n = p // PAGE + 1
            page = self.table[b, :n]
            ok = (page >= 0) & (page < len(self.units))
            at = np.where(ok, page, 0)
            for h in range(self.hkv):
                s = W.scores(q[r, h * g:(h + 1) * g], self.bounds[at, h, 0], self.bounds[at, h, 1], self.units[at, h])
                out[r, h] = W.choose(np.where(ok, s, -np.inf), n, budget, sink, recent)
        return out

    def check(self, q, task, pos, budget, sink=0, recent=0, max_len=0, live=None):
        out = torch.full((len(task), self.hkv, budget), -77, dtype=torch.int32, device="cuda")
        bounds = torch.from_numpy(self.bounds).cuda(), torch.from_numpy(self.units).cuda()
        self.kv.select_blocks(rows_to_dev(q), dev(task), dev(pos), bounds, budget, sink, recent, max_len, out=out)
        task = np.where(live, task, -1) if live is not None else task
        want = self.expect(q, task, pos, budget, sink, recent)
        got = out.cpu().numpy()
        assert np.array_equal(got, want), np.argwhere((got != want).any(2))[:5]


SHAPES = [(1, 1, 64), (2, 1, 128), (3, 1, 64), (8, 2, 64), (10, 2, 128), (28, 4, 128), (32, 2, 64), (9, 1, 128), (8, 8, 128)]


@pytest.mark.parametrize("hq,hkv,d", SHAPES)
@pytest.mark.parametrize("budget,sink,recent", [(1, 0, 0), (5, 1, 2), (8, 0, 8), (40, 2, 1)])
def test_choice_of_decode_rows(hq, hkv, d, budget, sink, recent):
    lens = [1, 16, 17, 80, 81, 97, 640, 641, 1100, 3000]
    c = Choice(hq + d + budget, lens, hq, hkv, d)
    c.check(c.queries(len(lens)), np.arange(len(lens)), np.array(lens) - 1, budget, sink, recent)


@pytest.mark.parametrize("hq,hkv,d", SHAPES)
def test_choice_of_many_rows_a_task(hq, hkv, d):
    """More rows than tasks: rows of a task together, alone, and out of order, with padding between."""
    lens = [700, 300, 45]
    c = Choice(hq + d, lens, hq, hkv, d)
    task = np.concatenate((np.zeros(70, int), np.full(5, 1), np.full(9, 2), c.rng.integers(0, 3, 60)))
    pos = np.array([c.rng.integers(0, lens[b]) for b in task])
    pos[:70] = np.arange(630, 700)
    for i, (t, p) in ((3, (-1, 5)), (72, (1, -1)), (80, (3, 4)), (100, (0, 2**31 - 1)), (101, (2**31 - 1, 0))):
        task[i], pos[i] = t, p
    live = (task >= 0) & (task < 3) & (pos >= 0) & (pos < 2**30)
    c.check(c.queries(len(task)), task, pos, 12, 1, 2, live=live)


def test_choice_of_equal_scores():
    """A handful of different pages: whole classes of equal scores at the border."""
    c = Choice(5, [9000, 20000, 200000], 8, 2, 64, pool=5)
    for budget in (7, 100, 400):
        c.check(c.queries(3), np.arange(3), np.array(c.lens) - 1, budget, 2, 3)
    c.bounds[:] = 3
    c.units[:] = -6
    c.check(c.queries(3), np.arange(3), np.array(c.lens) - 1, 50, 0, 1)  # all equal: the first ones


def test_choice_in_very_long_contexts():
    """More blocks than the workgroup's threads hold at once."""
    c = Choice(6, [16 * 9001, 16 * 20000 + 5], 4, 1, 64, pool=3000)
    for budget in (33, 2000):
        c.check(c.queries(2), [0, 1], np.array(c.lens) - 1, budget, 1, 1)


def test_choice_with_odd_numbers():
    """Pages that are not finite, page ids out of range, queries that are zero, not finite or extreme, units
    at both ends of their range."""
    lens = [900] * 8
    c = Choice(7, lens, 16, 2, 128)
    c.units[c.rng.random(c.units.shape) < 0.1] = 127
    c.units[c.rng.random(c.units.shape) < 0.1] = -120
    c.units[c.rng.random(c.units.shape) < 0.1] = 122
    c.table[c.rng.random(c.table.shape) < 0.1] = -4
    c.table[c.rng.random(c.table.shape) < 0.1] = len(c.units)
    c.table[2] = 2**31 - 1
    c.kv.set_block_table(c.table)
    q = c.queries(8)
    q[0] = 0.0
    q[1, 3, 5], q[1, 4, 6], q[2, 8, 0] = np.nan, np.inf, -np.inf
    q[3, 0:8] = np.nan
    q[4] *= 2.0 ** 110
    q[5] *= 2.0 ** -120
    q[6, :, 0] = float.fromhex("0x1.fep127")
    c.check(q, np.arange(8), np.array(lens) - 1, 20, 1, 2)
    c.check(q, np.arange(8), np.array(lens) - 1, 3, 0, 0)


def test_choice_up_to_max_len():
    c = Choice(8, [500, 400, 300], 8, 2, 64)
    pos = np.array([399, 398, 299])
    for max_len in (0, 500, 399, 299):
        c.check(c.queries(3), np.arange(3), pos, 4, 1, 1, max_len, live=pos < (max_len or 10**9))


@pytest.mark.parametrize("many", [False, True])
def test_choice_of_contexts_within_the_budget_and_beyond(many):
    """Rows whose blocks are all taken beside rows that choose; one row a task, and many."""
    lens = [16, 150, 176, 177, 160, 1700, 161, 700]
    c = Choice(10, lens, 8, 2, 128)
    task = np.arange(8) if not many else c.rng.integers(0, 8, 70)
    pos = np.array(lens)[task] - 1
    c.check(c.queries(task.size), task, pos, 10, 1, 2)
    c.check(c.queries(task.size), task, pos, 11, 0, 0)


def test_choice_in_rounds():
    """A table so wide that the rows' scores go through the workspace in rounds."""
    c = Choice(9, [1000, 700], 8, 8, 64)
    wide = np.full((2, 1 << 20), 2**31 - 1, np.int32)
    wide[:, :c.table.shape[1]] = c.table
    c.table = wide
    c.kv.set_block_table(wide)
    n = 21  # rounds of 8 rows
    assert tide.tide_rows_workspace_size(tide.TIDE_OP_BLOCK_SELECT, n, c.kv.dims, max_len=1 << 24) == (256 << 20) + 256
    task = c.rng.integers(0, 2, n)
    c.check(c.queries(n), task, np.array([c.rng.integers(300, c.lens[b]) for b in task]), 10, 1, 1)


def test_choice_of_many_tasks_with_a_few_rows_each():
    """Enough rows that workgroups walk several tasks, in rounds too."""
    rng = np.random.default_rng(19)
    lens = list(rng.integers(60, 400, 260))
    c = Choice(19, lens, 8, 2, 64)
    task = np.repeat(np.arange(260), 4)
    c.check(c.queries(task.size), task, np.array([rng.integers(50, lens[b]) for b in task]), 7, 1, 1)
    wide = np.full((260, 1 << 15), 2**31 - 1, np.int32)  # 256 KB of scores a row: rounds of 1,024 rows
    wide[:, :c.table.shape[1]] = c.table
    c.table = wide
    c.kv.set_block_table(wide)
    assert tide.tide_rows_workspace_size(tide.TIDE_OP_BLOCK_SELECT, task.size, c.kv.dims, max_len=1 << 19) == (256 << 20) + 256
    c.check(c.queries(task.size), task, np.array([rng.integers(50, lens[b]) for b in task]), 7, 0, 2)


# ---- attention over lists -----------------------------------------------------------------------------

class Sparse:
    def __init__(self, seed, lens, hq, hkv, d, scale=1.0):
        self.rng = rng = np.random.default_rng(seed)
        self.lens, self.hq, self.hkv, self.d = lens, hq, hkv, d
        self.table, pages = make_table(rng, lens)
        self.p = Pools(rng, pages, hq, hkv, d, self.table, scale)
        # past each context: what attention must not read
        for b, n in enumerate(lens):
            if n % PAGE:
                self.p.k[self.table[b, n // PAGE], :, n % PAGE:] = np.nan
                self.p.v[self.table[b, n // PAGE], :, n % PAGE:] = np.inf
        self.upload()

    def upload(self):
        self.p.kv.k_pool.copy_(rows_to_dev(self.p.k))
        self.p.kv.v_pool.copy_(rows_to_dev(self.p.v))
        self.p.kv.set_block_table(self.table)

    def rows(self, n):
        task = self.rng.integers(0, len(self.lens), n)
        pos = np.array([self.rng.integers(0, self.lens[b]) for b in task])
        return R.bf16(self.rng.standard_normal((n, self.hq, self.d))), task, pos

    def lists(self, task, pos, budget):
        """Distinct blocks in any order, -1 and blocks past the position among them."""
        sel = np.full((len(task), self.hkv, budget), -1)
        for r, p in enumerate(pos):
            n = p // PAGE + 1
            for h in range(self.hkv):
                pick = self.rng.permutation(np.arange(n + 3))[: self.rng.integers(1, budget + 1)]
                sel[r, h, self.rng.permutation(budget)[: pick.size]] = pick
        return sel

    def check(self, q, task, pos, sel, want_lse=True, live=None, only=None):
        n, g = len(task), self.hq // self.hkv
        out = torch.full((n, self.hq, self.d), 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((n, self.hq), 7.0, device="cuda") if want_lse else None
        self.p.kv.sparse(rows_to_dev(q), dev(task), dev(pos), dev(sel), out=out, lse=lse)
        got, got_lse = host(out), None if lse is None else host(lse)
        for r in range(n) if only is None else only:
            if live is not None and not live[r]:
                assert (got[r] == 7.0).all() and (lse is None or (got_lse[r] == 7.0).all())
                continue
            for h in range(self.hkv):
                at, gs = [b for b in sel[r, h] if 0 <= b <= pos[r] // PAGE], slice(h * g, (h + 1) * g)
                at = [b for b in at if 0 <= self.table[task[r], b] < len(self.p.k)]
                page = self.table[task[r], : pos[r] // PAGE + 1]
                page = np.where((page >= 0) & (page < len(self.p.k)), page, 0)
                k, v = (x[page, h].reshape(-1, self.d) for x in (self.p.k, self.p.v))
                o, z, spread, size = W.attend(q[r, gs], k, v, at, pos[r], float(np.float32(self.d ** -0.5)))
                # a score off by e changes a weight by a factor of about 1 + e, and the sum that divides it
                e = R.score_bound(self.d, size)
                worst = (np.abs(got[r, gs] - o) - R.out_bound(o, spread) - 2 * e * spread).max()
                assert worst <= 0, (r, h, worst)
                if lse is not None and at:
                    assert np.abs(got_lse[r, gs] - z).max() <= e + 2.0 ** -22 * np.abs(z).max()
                elif lse is not None:
                    assert (got_lse[r, gs] == -np.inf).all() and (got[r, gs] == 0).all()


@pytest.mark.parametrize("hq,hkv,d", SHAPES + [(64, 8, 128), (16, 1, 128)])
@pytest.mark.parametrize("budget", [1, 2, 7, 33])
def test_attention_over_lists(hq, hkv, d, budget):
    s = Sparse(hq + d + budget, [1, 15, 16, 17, 100, 500, 900], hq, hkv, d)
    q, task, pos = s.rows(24)
    pos[:7], task[:7] = np.array(s.lens) - 1, np.arange(7)
    s.check(q, task, pos, s.lists(task, pos, budget), want_lse=budget != 7)


@pytest.mark.parametrize("rows,budget", [(1, 200), (1, 1001), (3, 300), (40, 520), (300, 130)])
def test_attention_over_long_lists(rows, budget):
    """Lists that are split over workgroups and joined, and lists longer than a workgroup's batch."""
    s = Sparse(budget, [16 * 1200, 5000], 8, 2, 128)
    q, task, pos = s.rows(rows)
    pos[0], task[0] = s.lens[0] - 1, 0
    sel = s.lists(task, pos, budget)
    sel[0, :, :] = s.rng.permutation(1200)[:budget]
    s.check(q, task, pos, sel)


@pytest.mark.parametrize("hq,hkv,d", [(8, 8, 128), (14, 2, 64)])
def test_attention_of_a_row_a_task(hq, hkv, d):
    """A decode batch: as many tasks as rows, too many to split."""
    n = 300 if hkv < 8 else 70
    s = Sparse(21, list(np.random.default_rng(21).integers(1, 700, n)), hq, hkv, d)
    q, _, _ = s.rows(n)
    task, pos = np.arange(n), np.array(s.lens) - 1
    s.check(q, task, pos, s.lists(task, pos, 11))


@pytest.mark.parametrize("hq,hkv", [(32, 4), (1, 1), (4, 2), (16, 1)])
@pytest.mark.parametrize("budget", [1, 2, 40, 192])
def test_rows_taken_together(hq, hkv, budget):
    """Runs of rows of one task whose lists overlap much, little and not at all, with rows of other tasks and
    padding between; enough of them that none is split."""
    s = Sparse(hq + budget, [4000, 700, 3300], hq, hkv, 128)
    n = 600 // hkv
    q, task, pos = s.rows(n)
    task[: n // 2], pos[: n // 2] = 0, 3400 + np.arange(n // 2)
    sel = s.lists(task, pos, budget)
    for r in range(n // 2):  # neighbours differ in a few blocks; each has its own last one
        common = np.random.default_rng(r // 16).permutation(200)[:budget]
        sel[r] = common
        own = s.rng.permutation(np.setdiff1d(np.arange(212), common))[: budget // 8]
        sel[r, :, : own.size] = own
        sel[r, :, budget - 1] = pos[r] // PAGE
    live = np.ones(n, bool)
    for i, (t, p) in ((3, (-1, 9)), (17, (0, -4)), (n // 2 + 1, (3, 0))):
        task[i], pos[i], live[i] = t, p, False
    some = sorted(set(s.rng.permutation(n)[:60]) | set(range(20)) | {n // 2 + 1, n - 1})  # all are computed
    s.check(q, task, pos, sel, live=live, only=some)


def test_rows_taken_together_that_list_a_block_twice():
    s = Sparse(31, [3000], 8, 1, 64)
    q, task, pos = s.rows(600)
    pos[:] = 2000 + np.arange(600)
    sel = np.tile(np.arange(20), (600, 1, 1))
    sel[5, 0, 7] = 3           # block 3 twice in row 5 alone
    sel[64:72, 0, 1] = 0       # and in all rows of a group
    s.check(q, task, pos, sel, only=range(90))


def test_rows_taken_together_do_not_share_what_is_not_a_number():
    """V and K that are not finite in blocks that some rows of a group list, and past the position of some."""
    s = Sparse(32, [3000], 8, 1, 128)
    q, task, pos = s.rows(600)
    pos[:] = 2000 + np.arange(600)
    sel = np.tile(np.arange(20), (600, 1, 1))
    sel[:, 0, 19] = pos // PAGE
    sel[2, 0, 4], sel[3, 0, 5], sel[9, 0, 6] = 40, 41, 42
    for b, x in ((40, np.nan), (41, np.inf), (42, -np.inf)):
        s.p.v[s.table[0, b], 0, 3, 5] = x
        s.p.k[s.table[0, b], 0, 9, 7] = x
    at = 2013  # position of row 13: rows 8 .. 12 of its group of 8 or 4 list the block and do not see it
    s.p.v[s.table[0, at // PAGE], 0, at % PAGE, 1] = np.inf
    s.upload()
    out = host(s.p.kv.sparse(rows_to_dev(q), dev(task), dev(pos), dev(sel)))
    bad = {r for r in range(600) if not np.isfinite(out[r]).all()}
    assert bad == {2, 3, 9} | {r for r in range(13, 600) if pos[r] // PAGE == at // PAGE}
    s.check(q, task, pos, sel, want_lse=False, only=[0, 1, 4, 8, 10, 12, 40, 599])


@pytest.mark.parametrize("budget", [300, 900])
def test_lists_too_long_to_take_rows_together(budget):
    s = Sparse(33, [16 * 1000], 8, 1, 128)
    q, task, pos = s.rows(600)
    sel = s.lists(task, pos, budget)
    s.check(q, task, pos, sel, only=range(0, 600, 29))


def test_rows_that_see_nothing_and_padding():
    """Empty lists give zeros and -inf; padding rows stay as they are."""
    s = Sparse(3, [200, 40], 28, 4, 128)
    for rows in (9, 700):  # split and not
        q, task, pos = s.rows(rows)
        sel = s.lists(task, pos, 32)
        sel[1], sel[2, 1:], sel[3] = -1, -5, pos[3] // PAGE + 1
        sel[4, 0], sel[4, 0, 31] = -1, 0
        live = np.ones(rows, bool)
        for i, (t, p) in ((0, (-1, 0)), (5, (2, 0)), (6, (0, -1)), (7, (0, 2**31 - 1))):
            task[i], pos[i], live[i] = t, p, False
        s.check(q, task, np.where(live, pos, pos), sel, live=live)


def test_attention_with_bad_pages(monkeypatch):
    s = Sparse(4, [300, 500], 8, 2, 64)
    q, task, pos = s.rows(20)
    sel = s.lists(task, pos, 12)
    s.table[0, ::3], s.table[1, 1::4] = -1, len(s.p.k)
    s.upload()
    s.check(q, task, pos, sel)
    monkeypatch.setenv("TIDE_DEBUG_CHECKS", "1")
    with pytest.raises(tide.TideError) as e:
        s.check(q, task, pos, sel)
    assert e.value.status == tide.TIDE_ERR_PAGE_RANGE


def test_a_block_listed_twice_counts_twice():
    s = Sparse(5, [100], 8, 2, 64)
    q, task, pos = s.rows(4)
    pos[:] = 99
    s.check(q, task, pos, np.tile([3, 0, 3, -1, 3], (4, 2, 1)))


def test_large_scores_and_values():
    """Weights that all but one key lose, maxima that keep rising, and scores far below zero."""
    s = Sparse(6, [800], 4, 1, 128, scale=30.0)
    q, task, pos = s.rows(6)
    q *= 4.0
    pos[:] = 799
    s.check(q, task, pos, np.tile(np.arange(50), (6, 1, 1)))
    s.p.k[...] = -np.abs(s.p.k)
    s.upload()
    s.check(np.abs(q), task, pos, np.tile(np.arange(50), (6, 1, 1)))


@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 128), (16, 2, 64)])
def test_large_scores_of_rows_taken_together(hq, hkv, d):
    """The same for rows of one task, whose lists differ, so that their maxima rise at different blocks."""
    s = Sparse(7, [1600], hq, hkv, d, scale=20.0)
    s.p.k *= (2.0 ** (np.arange(s.p.k.shape[0]) % 4))[:, None, None, None]
    s.upload()
    q, task, pos = s.rows(600)
    pos[:] = 1000 + np.arange(600)
    sel = s.lists(task, pos, 30)
    sel[:, :, 0] = pos[:, None] // PAGE
    for r in range(600):  # (distinct blocks, the last one first)
        for h in range(hkv):
            sel[r, h, 1:][sel[r, h, 1:] == sel[r, h, 0]] = -1
    s.check(q, task, pos, sel, only=range(0, 600, 7))


def test_keys_that_are_not_numbers_reach_the_rows_that_list_them():
    s = Sparse(7, [200], 8, 2, 64)
    q, task, pos = s.rows(3)
    pos[:] = 199
    s.p.k[s.table[0, 4], 0, 3, 5] = np.nan
    s.p.v[s.table[0, 6], 1, 3, 5] = np.nan
    s.upload()
    sel = np.tile([0, 1, 2, 4], (3, 2, 1))
    sel[1:, 0], sel[2:, 1] = [0, 1, 2, 3], [0, 1, 2, 6]
    out = host(s.p.kv.sparse(rows_to_dev(q), dev(task), dev(pos), dev(sel)))
    assert np.isnan(out[0, :4]).all() and np.isfinite(out[0, 4:]).all() and np.isfinite(out[1]).all()
    assert np.isfinite(out[2, :4]).all() and np.isnan(out[2, 4:, 5]).all()
    assert np.isfinite(np.delete(out[2, 4:], 5, axis=1)).all()


# ---- together ------------------------------------------------------------------------------------------

HQ, HKV, D, BUDGET, SINK, RECENT = 28, 4, 128, 6, 1, 2


def step(kv, table, want, rows, q, k, v, bounds):
    """One step of a rollout engine without a length from the host."""
    table.map(want, rows)
    kv.append_slots(k, v, rows[2], bounds)
    sel = kv.select_blocks(q, rows[0], rows[1], bounds, BUDGET, SINK, RECENT)
    lse = torch.zeros((q.shape[0], HQ), device="cuda")
    return sel, kv.sparse(q, rows[0], rows[1], sel, out=torch.zeros_like(q), lse=lse), lse


def engine(tasks, pages_per_task, pages):
    table = tide.PageTable(tasks, pages_per_task, pages)
    kv = tide.PagedKV(pages, HQ, HKV, D, table.block_table.cpu().numpy())
    kv.block_table = table.block_table
    return kv, table, kv.new_bounds()


def normal(rng, *shape):
    return rows_to_dev(rng.standard_normal(shape))


def test_a_run_of_steps():
    """Observations and tokens come in, tasks end and their pages go to others: bounds, choices and outputs
    after every step against the definitions on the host's own copy of every context."""
    rng = np.random.default_rng(11)
    n = 3
    kv, table, bounds = engine(n, 20, 40)
    ctx = [[np.zeros((0, HKV, D))] * 2 for _ in range(n)]
    lens = np.zeros(n, int)
    for new in ([200, 37, 5], [1, 1, 1], [1, 60, 1], [0, -97, 130], [1, 40, 1], [1, 1, 1]):
        want = lens + new
        e = np.maximum(0, new)
        total = int(e.sum())
        rows = table.new_rows(total + 2)  # some padding
        q, k, v = normal(rng, total + 2, HQ, D), normal(rng, total + 2, HKV, D), normal(rng, total + 2, HKV, D)
        sel, out, lse = step(kv, table, dev(want), rows, q, k, v, bounds)
        start = np.concatenate(([0], np.cumsum(e)))
        assert np.array_equal(table.row_start.cpu().numpy(), start) and np.array_equal(table.lens.cpu().numpy(), want)
        for b in range(n):
            at = slice(start[b], start[b + 1])
            ctx[b] = [np.concatenate((c[: want[b]], host(x)[at]))[: want[b]] for c, x in zip(ctx[b], (k, v))]
        bt, hb, hu = table.block_table.cpu().numpy(), bounds[0].cpu().numpy(), bounds[1].cpu().numpy()
        for b in range(n):
            for i in range(max(0, lens[b] if new[b] > 0 else want[b]) // PAGE, W.pages_of(want[b])):
                if new[b] <= 0:
                    continue  # a page that was cut keeps the bounds of what it held
                for h in range(HKV):
                    hi, lo, s = W.bounds_of(ctx[b][0][PAGE * i: PAGE * (i + 1), h])
                    assert hu[bt[b, i], h] == s and np.array_equal(hb[bt[b, i], h], np.stack((hi, lo)))
        hq, hsel, hout, hlse = host(q), sel.cpu().numpy(), host(out), host(lse)
        g = HQ // HKV
        for r in range(total):
            b = int(np.searchsorted(start, r, side="right") - 1)
            pos = lens[b] + r - start[b]
            if pos < want[b] - 4 and r % 7:
                continue  # the ends of observations, and a part of the rest
            for h in range(HKV):
                gs, page = slice(h * g, (h + 1) * g), bt[b, : pos // PAGE + 1]
                s = W.scores(hq[r, gs], hb[page, h, 0], hb[page, h, 1], hu[page, h])
                assert hsel[r, h].tolist() == W.choose(s, pos // PAGE + 1, BUDGET, SINK, RECENT)
                o, z, spread, size = W.attend(hq[r, gs], ctx[b][0][:, h], ctx[b][1][:, h], hsel[r, h], pos,
                                              float(np.float32(D ** -0.5)))
                e_ = R.score_bound(D, size)
                assert (np.abs(hout[r, gs] - o) <= R.out_bound(o, spread) + 2 * e_ * spread).all()
                assert np.abs(hlse[r, gs] - z).max() <= e_ + 2.0 ** -22 * np.abs(z).max()
        assert (hout[total:] == 0).all() and (hlse[total:] == 0).all()
        lens = want


def test_a_captured_step_goes_on_as_contexts_grow():
    """One graph of map, append, choice and attention, replayed for 40 tokens with eager work between,
    against the same steps made eagerly: the same bits."""
    n = 5
    first = [3, 90, 16, 31, 200]
    gen = np.random.default_rng(12)
    prompt = [normal(gen, sum(first), x, D) for x in (HQ, HKV, HKV)]
    tokens = [[normal(gen, n, x, D) for x in (HQ, HKV, HKV)] for _ in range(40)]

    def begin():
        kv, table, bounds = engine(n, 20, 70)
        step(kv, table, dev(first), table.new_rows(sum(first)), *prompt, bounds)
        return kv, table, bounds

    kv, table, bounds = begin()
    want = []
    for t in tokens:
        rows = table.new_rows(n)
        want.append(step(kv, table, table.lens + 1, rows, *t, bounds) + (rows[2],))
    final = [x.clone() for x in (kv.k_pool, kv.v_pool, *bounds, table.block_table, table.lens, table.free_count)]

    kv, table, bounds = begin()
    buf = [torch.zeros_like(x) for x in tokens[0]]
    rows = table.new_rows(n)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = step(kv, table, table.lens + 1, rows, *buf, bounds)
    torch.cuda.synchronize()
    assert table.lens.tolist() == first
    for i, t in enumerate(tokens):
        for b, x in zip(buf, t):
            b.copy_(x)
        graph.replay()
        for a, b in zip(got + (rows[2],), want[i]):
            assert torch.equal(a, b), i
        torch.zeros(1000, device="cuda").sum().item()
    for a, b in zip((kv.k_pool, kv.v_pool, *bounds, table.block_table, table.lens, table.free_count), final):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_another_stream():
    rng = np.random.default_rng(13)
    results = []
    for side in (False, True):
        rng = np.random.default_rng(13)
        kv, table, bounds = engine(2, 20, 40)
        args = [normal(rng, 130, x, D) for x in (HQ, HKV, HKV)]
        torch.cuda.synchronize()
        s = torch.cuda.Stream() if side else torch.cuda.current_stream()
        with torch.cuda.stream(s):
            results.append(step(kv, table, dev([30, 100]), table.new_rows(130), *args, bounds))
        torch.cuda.synchronize()
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_pools_past_32_bits():
    """Pages, slots and bounds whose offsets do not fit in 32 bits: what a small pool gives."""
    rng = np.random.default_rng(16)
    small, far = 41, 2_200_000
    lens = [300, 33, 270]
    table = np.stack((np.arange(19), np.arange(38, 57) % small, np.arange(19, 38))).astype(np.int32)
    spread = np.concatenate((np.arange(0, 10), rng.permutation(np.arange(far - 200, far))[: small - 10])).astype(np.int32)
    task, pos = np.repeat([0, 2], 40), np.concatenate((np.arange(260, 300), np.arange(230, 270)))
    hq, hkv, d = 8, 2, 128  # K of 18 GB, bounds of 1.1 GB and then of 4.6 GB
    k, v, q = normal(rng, 80, hkv, d), normal(rng, 80, hkv, d), normal(rng, 80, hq, d)
    fill_k, fill_v = normal(rng, small, hkv, PAGE, d), normal(rng, small, hkv, PAGE, d)
    results = []
    for pages, at in ((small, np.arange(small, dtype=np.int32)), (far, spread)):
        bt = at[table]
        kv = tide.PagedKV(pages, hq, hkv, d, bt, fill_canary=False)
        ids = dev(at, np.int64)
        kv.k_pool[ids], kv.v_pool[ids] = fill_k, fill_v
        bounds = kv.new_bounds()
        kv.key_bounds(dev(lens), bounds)
        slot = bt[task, pos // PAGE].astype(np.int64) * PAGE + pos % PAGE
        kv.append_slots(k, v, dev(slot, np.int64), bounds)
        sel = kv.select_blocks(q, dev(task), dev(pos), bounds, 5, 1, 1)
        few = kv.select_blocks(q[[39, 79]], dev([0, 2]), dev([299, 269]), bounds, 5, 1, 1)
        results.append([kv.k_pool[ids], kv.v_pool[ids], bounds[0][ids], bounds[1][ids], sel, few,
                        kv.sparse(q, dev(task), dev(pos), sel), kv.sparse(q[[39, 79]], dev([0, 2]), dev([299, 269]), few)])
        if pages == far:  # the bounds again, four times as far apart
            wide = tide.PagedKV(1, hq, hkv, d, 4 * bt, fill_canary=False)
            b = [torch.empty((4 * far,) + x.shape[1:], dtype=torch.int8, device="cuda") for x in bounds]
            for x, y in zip(b, bounds):
                x[4 * ids] = y[ids]
            for rows, s in ((slice(None), sel), ([39, 79], few)):
                assert torch.equal(wide.select_blocks(q[rows], dev(task[rows]), dev(pos[rows]), b, 5, 1, 1), s)
            del wide, b
        del kv, bounds
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_two_steps_at_once():
    """Two engines on streams of their own, without a wait between them: what each gives alone."""
    def make(seed):
        rng = np.random.default_rng(seed)
        return engine(2, 20, 40), [[normal(rng, e, x, D) for x in (HQ, HKV, HKV)] for e in (250, 2, 2, 60)]

    wants = [[150, 100], [151, 101], [152, 102], [202, 112]]
    alone, both = [], []
    for seed in (17, 18):
        (kv, table, bounds), args = make(seed)
        alone.append([step(kv, table, dev(w), table.new_rows(a[0].shape[0]), *a, bounds) for w, a in zip(wants, args)])
    engines = [make(17), make(18)]
    w = [dev(x) for x in wants]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in engines]
    both = [[], []]
    for i in range(len(wants)):
        for j, ((kv, table, bounds), args) in enumerate(engines):
            with torch.cuda.stream(streams[j]):
                both[j].append(step(kv, table, w[i], table.new_rows(args[i][0].shape[0]), *args[i], bounds))
    torch.cuda.synchronize()
    for a, b in zip(alone, both):
        for x, y in zip(a, b):
            assert all(torch.equal(m, n) for m, n in zip(x, y))


def test_bounds_after_other_appends():
    """Contexts that the host-planned calls wrote: their bounds are those of an append by slots."""
    rng = np.random.default_rng(14)
    kv, table, bounds = engine(2, 20, 40)
    rows = table.new_rows(333)
    table.map(dev([33, 300]), rows)
    k, v = normal(rng, 333, HKV, D), normal(rng, 333, HKV, D)
    kv.append_slots(k, v, rows[2], bounds)
    other = tide.PagedKV(40, HQ, HKV, D, table.block_table.cpu().numpy())
    other.append(k, v, [0, 0], [33, 300])
    assert torch.equal(other.k_pool.view(torch.int16), kv.k_pool.view(torch.int16))
    again = other.key_bounds(table.lens, other.new_bounds())
    assert torch.equal(again[0], bounds[0]) and torch.equal(again[1], bounds[1])


def test_all_blocks_is_decode():
    """A budget that holds every block: the decode of whole contexts, within both sides' roundings."""
    rng = np.random.default_rng(15)
    kv, table, bounds = engine(2, 20, 40)
    step(kv, table, dev([33, 300]), table.new_rows(333), normal(rng, 333, HQ, D), normal(rng, 333, HKV, D),
         normal(rng, 333, HKV, D), bounds)
    q = normal(rng, 2, HQ, D)
    task, pos = dev([0, 1]), dev([32, 299])
    sel = kv.select_blocks(q, task, pos, bounds, 20)
    assert sel[0, 0].tolist() == [0, 1, 2] + [-1] * 17 and sel[1, 3].tolist() == list(range(19)) + [-1]
    a, b = host(kv.sparse(q, task, pos, sel)), host(kv.decode(q, [33, 300]))
    assert np.abs(a - b).max() <= 4 * 2.0 ** -8 * max(1.0, np.abs(b).max())
