"""The references of page maps, key bounds and block choice, checked on the CPU against facts that do not
come from them; planted mistakes must show."""
import numpy as np
import pytest

import cache_reference as R
import rows_reference as W


def test_a_page_belongs_to_one_task_and_none_is_lost():
    rng = np.random.default_rng(3)
    n, stride, pool = 9, 12, 40
    table, free, count = np.zeros((n, stride), int), np.arange(pool), pool
    lens = [0] * n
    refused = 0
    for _ in range(200):
        want = [int(x) for x in rng.integers(0, stride * 16 + 1, n)]
        total = sum(max(0, w - a) for a, w in zip(lens, want))
        out, table, free, count, start, rows = W.page_map(lens, want, table, free, count, total + 3)
        held = [table[b, i] for b in range(n) for i in range(W.pages_of(out[b]))]
        assert sorted(held + list(free[:count])) == list(range(pool))
        assert start[-1] <= total and (rows[start[-1]:] == -1).all()
        for b in range(n):
            mine = rows[start[b]:start[b + 1]]
            assert out[b] in (lens[b], want[b])
            if out[b] != want[b]:
                refused += 1
                assert (mine == -1).all()
            for j, (task, pos, slot) in enumerate(mine[mine[:, 0] >= 0]):
                assert (task, pos) == (b, lens[b] + j) and slot == table[b, pos // 16] * 16 + pos % 16
        lens = out
    assert refused


def test_refusals_by_rows_and_pages():
    table = [[5, 9, 9], [6, 9, 9], [7, 9, 9]]
    out, t, free, top, start, rows = W.page_map([10, 16, 3], [20, 17, 4], table, [1, 2], 1, 12)
    assert out == [20, 16, 4] and top == 0 and t[0, 1] == 1 and t[1, 1] == 9  # one page: the first task's
    assert start == [0, 10, 11, 12] and rows[10].tolist() == [-1, -1, -1] and rows[11].tolist() == [2, 3, 7 * 16 + 3]
    out, t, free, top, start, rows = W.page_map([10, 16, 3], [20, 17, 4], table, [1, 2], 2, 10)
    assert out == [20, 16, 3] and top == 1 and start == [0, 10, 10, 10]       # no rows behind the first task
    out, *_ = W.page_map([10, 16, 3], [49, -1, 0], table, [1, 2], 2, 100)
    assert out == [10, 16, 0]                                                # lengths that are none


def test_bounds_hold_every_key_and_are_tight():
    rng = np.random.default_rng(5)
    for _ in range(200):
        k = R.bf16(rng.standard_normal((rng.integers(1, 17), 64)) * 2.0 ** rng.integers(-100, 100))
        hi, lo, s = W.bounds_of(k)
        f = 2.0 ** s
        assert (lo * f <= k).all() and (k <= hi * f).all() and np.abs([hi, lo]).max() <= 127
        assert ((hi - 1) * f < k.max(0)).all() and ((lo + 1) * f > k.min(0)).all()
        assert np.abs(k).max() > 63.5 * f  # half the unit would not do


def test_a_score_bounds_every_key_of_its_page():
    rng = np.random.default_rng(6)
    for _ in range(50):
        k = R.bf16(rng.standard_normal((16, 64)))
        q = R.bf16(rng.standard_normal((4, 64)) * 2.0 ** rng.integers(-3, 4, (4, 1)))
        hi, lo, s = W.bounds_of(k)
        code, t = W.codes_of(q)
        assert np.abs(code * 2.0 ** t[:, None] - q).max() <= 0.5 * 2.0 ** t.max()
        best = ((code * 2.0 ** t[:, None]) @ k.T).max()
        assert W.scores(q, hi[None], lo[None], np.array([s]))[0] >= best


@pytest.mark.parametrize("blocks,want", [(3, [0, 1, 2, -1]), (4, [0, 1, 2, 3]), (6, [0, 2, 4, 5]), (7, [0, 2, 4, 6])])
def test_choice(blocks, want):
    assert W.choose([9, 1, 5, 1, 5, 5, 0], blocks, 4, 1, 1) == want


def test_choice_among_equals_and_infinities():
    assert W.choose([0.0] * 9, 9, 3, 0, 0) == [0, 1, 2]
    assert W.choose([0, -np.inf, np.inf, 1, np.inf, 0], 6, 2, 0, 0) == [2, 4]
    assert W.choose([1, 2, 3, 4], 4, 2, 1, 1) == [0, 3]


def test_attention_of_all_blocks_is_attention():
    rng = np.random.default_rng(7)
    q, k, v = (rng.standard_normal(x) for x in ((1, 4, 64), (40, 1, 64), (40, 1, 64)))
    o, z, _, _ = R.attention(q, k, v, 39, 0.125)
    got, lse, _, _ = W.attend(q[0], k[:, 0], v[:, 0], [2, 0, -1, 1, 5], 39, 0.125)
    assert np.allclose(got, o[0], atol=1e-12) and np.allclose(lse, z[0], atol=1e-12)
    none = W.attend(q[0], k[:, 0], v[:, 0], [-1, 3], 39, 0.125)
    assert (none[0] == 0).all() and (none[1] == -np.inf).all()
