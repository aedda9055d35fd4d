"""Ways through the choice of blocks and the attention over lists that sizes and values decide (needs an MI355X): odd
values where rows go task by task, many (row, kv head) pairs over long contexts, and the widest tables whose rows are taken
together."""
import numpy as np
import pytest
import torch

import cache_reference as R
import paper_2608_10402_amd as tide
import rows_reference as W
from test_gpu_rows import Choice, Sparse, dev, rows_to_dev

pytestmark = pytest.mark.gpu

PAGE = 16


# ---- the choice, many rows a task ------------------------------------------------------------------------

@pytest.mark.parametrize("hq,hkv,d", [(16, 2, 128), (8, 8, 64), (16, 1, 64), (6, 2, 128), (4, 1, 64)])
def test_choice_with_odd_numbers_of_many_rows_a_task(monkeypatch, hq, hkv, d):
    """Units at both ends of their range and of keys that are not finite, page ids out of range, queries that are
    zero, not finite or extreme: in some tasks, and rows of the others beside them."""
    lens = [900, 1800, 2500, 700, 1300, 900]
    c = Choice(hq + d, lens, hq, hkv, d)
    odd = np.unique(np.concatenate([c.table[b, : W.pages_of(lens[b])] for b in (0, 1)]))
    for unit in (127, -120, 122, 41, -41):
        some = odd[c.rng.random(odd.size) < 0.15]
        c.units[some] = np.where(c.rng.random((some.size, hkv)) < 0.5, unit, c.units[some])
    good = c.table.copy()
    for b in (0, 2):
        c.table[b][c.rng.random(c.table.shape[1]) < 0.1] = -4
        c.table[b][c.rng.random(c.table.shape[1]) < 0.1] = len(c.units)
    c.table[3] = 2**31 - 1
    c.kv.set_block_table(c.table)
    n = 34 * len(lens)  # (task by task from 16 rows a task on)
    task = np.repeat(np.arange(len(lens)), 34)
    pos = np.array([c.rng.integers(0, lens[b]) for b in task])
    pos[::34] = np.array(lens) - 1
    q = c.queries(n)
    q[2], q[70] = 0.0, 0.0
    q[5, 0, 5], q[6, -1, 6], q[41, 0, 0] = np.nan, np.inf, -np.inf
    q[7] = np.nan
    q[8:12] *= 2.0 ** 110
    q[12:16] *= 2.0 ** -120
    q[16, :, 0] = float.fromhex("0x1.fep127")
    q[105] *= 2.0 ** 70  # (a task of ordinary units)
    q[140] *= 2.0 ** -70
    q = R.bf16(q)
    for order in (np.arange(n), c.rng.permutation(n)):
        c.check(q[order], task[order], pos[order], 20, 1, 2)
        c.check(q[order], task[order], pos[order], 3, 0, 0)
    monkeypatch.setenv("TIDE_DEBUG_CHECKS", "1")
    with pytest.raises(tide.TideError) as e:
        c.check(q, task, pos, 20, 1, 2)
    assert e.value.status == tide.TIDE_ERR_PAGE_RANGE
    c.table = good
    c.kv.set_block_table(good)
    c.check(q, task, pos, 20, 1, 2)  # nothing out of range: no error


# ---- the choice, many pairs ------------------------------------------------------------------------------

class ManyPairs(Choice):
    """More than 1,024 (row, kv head) pairs over few different pages, whose scores are worked out once a page."""

    def expect(self, q, task, pos, budget, sink, recent):
        g = self.hq // self.hkv
        out = np.full((len(task), self.hkv, budget), -77)
        for r, (b, p) in enumerate(zip(task, pos)):
            at = self.table[b, : p // PAGE + 1]
            ok = (at >= 0) & (at < len(self.units))
            for h in range(self.hkv):
                s = W.scores(q[r, h * g:(h + 1) * g], self.bounds[:, h, 0], self.bounds[:, h, 1], self.units[:, h])
                out[r, h] = W.choose(np.where(ok, s[np.where(ok, at, 0)], -np.inf), at.size, budget, sink, recent)
        return out


LONG = [16 * 6144, 16 * 6144 + 1, 16 * 9001, 16 * 16385 + 7, 3000]  # around what threads hold, and above all bits


def many_pairs(seed, lens, pool):
    c = ManyPairs(seed, lens, 8, 8, 64, pool=pool)
    task = np.arange(130) % len(lens)
    return c, c.queries(130), task, np.array(lens)[task] - 1 - (np.arange(130) // len(lens)) % 16


@pytest.mark.parametrize("budget,sink,recent", [(33, 1, 1), (400, 0, 3), (2000, 2, 0), (5000, 0, 0)])
def test_choice_of_many_pairs_in_long_contexts(budget, sink, recent):
    c, q, task, pos = many_pairs(61, LONG, 3000)
    c.check(q, task, pos, budget, sink, recent)


@pytest.mark.parametrize("lens", [LONG, [9000, 20000, 2100, 640]])
@pytest.mark.parametrize("budget", [7, 100, 400])
def test_choice_of_many_pairs_with_equal_scores(lens, budget):
    c, q, task, pos = many_pairs(62, lens, 5)
    c.check(q, task, pos, budget, 2, 3)
    c.bounds[:] = 3
    c.units[:] = -6
    c.check(q, task, pos, budget, 0, 1)  # all equal: the first ones


@pytest.mark.parametrize("pool", [5, 700])
@pytest.mark.parametrize("budget", [6, 90, 1500])
def test_choice_of_many_pairs_with_infinite_scores(pool, budget):
    """Keys that are not finite and page ids out of range, fewer and more of them than the budget."""
    c, q, task, pos = many_pairs(63, LONG, pool)
    c.units[:: 5 if pool == 5 else 90] = 127
    c.table[c.rng.random(c.table.shape) < 0.05] = -1
    c.table[1, 40:] = pool  # few blocks that have a score
    c.kv.set_block_table(c.table)
    c.check(q, task, pos, budget, 1, 2)


# ---- attention over lists in wide tables -------------------------------------------------------------------

def wide(seed, d, stride):
    """600 rows at the end of a context that fills a table of `stride` pages, each a copy of one of 125."""
    s = Sparse(seed, [2000], 8, 1, d)
    s.table = s.rng.permutation(np.tile(s.table[0, :125], stride // 125 + 1))[None, :stride].astype(np.int32)
    s.upload()
    q, task, _ = s.rows(600)
    pos = PAGE * stride - 1 - np.arange(600)[::-1]
    common = s.rng.permutation(stride - 60)[:37]
    sel = np.full((600, 1, 40), -1)
    sel[:, 0, :37] = common
    sel[:, 0, 3] = stride - 50
    sel[:, 0, 38], sel[:, 0, 39] = stride - 1, pos // PAGE  # (the last block of all, past most rows' positions)
    sel[pos // PAGE == stride - 1, 0, 38] = -1
    own = s.rng.permutation(stride - 60)[:600]
    sel[::3, 0, 5] = np.where(np.isin(own, common), sel[:, 0, 5], own)[::3]
    return s, q, task, pos, sel


@pytest.mark.parametrize("d,most", [(64, 16384), (128, 32768)])  # blocks of a context that a workgroup can mark
@pytest.mark.parametrize("more", [0, 1])
def test_rows_of_the_widest_tables(d, most, more):
    s, q, task, pos, sel = wide(d + more, d, most + more)
    some = [0, 1, 583, 584, 599]
    s.check(q, task, pos, sel, only=some)
    out = s.p.kv.sparse(rows_to_dev(q), dev(task), dev(pos), dev(sel))
    few = s.p.kv.sparse(rows_to_dev(q[:400]), dev(task[:400]), dev(pos[:400]), dev(sel[:400]))  # one by one
    assert torch.isfinite(out).all()
    # each is off by at most 2^-8 of itself (the output's rounding) and sum_i w_i 2^-8 |v_i - o|, at most 2^-8 2 max|v|
    # (the weights', whose rounded sum divides)
    a, b = out[:400].double(), few.double()
    top = torch.tensor(np.abs(s.p.v).max(), device="cuda")
    assert ((a - b).abs() <= 2 * 2.0 ** -8 * (a.abs() + 2 * top)).all()


def test_bad_pages_of_rows_taken_together(monkeypatch):
    """Blocks whose page ids are out of range, in some rows' lists alone and in all of them."""
    s = Sparse(64, [3000], 8, 1, 128)
    s.table[0, [3, 7, 12]], s.table[0, 40], s.table[0, 50:60] = -1, len(s.p.k), 2**31 - 1
    s.upload()
    q, task, pos = s.rows(600)
    pos[:] = 2000 + np.arange(600)
    sel = np.tile(np.arange(20), (600, 1, 1))
    sel[5, 0, 0], sel[9, 0, 1] = 40, 55
    sel[24:28, 0] = np.arange(50, 70)  # (of which ten are there)
    sel[32, 0] = np.arange(50, 70) % 10 + 50
    sel[40:48, 0] = -1
    sel[44:46, 0, 7] = 52  # rows that list a bad block alone
    s.check(q, task, pos, sel, only=range(60))
    monkeypatch.setenv("TIDE_DEBUG_CHECKS", "1")
    with pytest.raises(tide.TideError) as e:
        s.check(q, task, pos, sel)
    assert e.value.status == tide.TIDE_ERR_PAGE_RANGE
    keep = np.tile(np.arange(20, 40), (600, 1, 1))
    s.check(q, task, pos, keep, only=range(9))  # none listed: no error
