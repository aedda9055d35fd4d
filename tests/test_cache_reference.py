"""The references of the 4-bit cache and of eviction, checked on the CPU against each other and
against facts that do not come from them; planted mistakes must show."""
import numpy as np
import pytest

import cache_reference as R


def test_rounding_is_nearest_within_the_scale():
    rng = np.random.default_rng(1)
    x = R.bf16(rng.standard_normal((200, 64)) * np.exp2(rng.integers(-20, 20, (200, 1))))
    code, scale = R.encode(x)
    y = R.decode(code, scale)
    f = np.repeat(2.0 ** (scale - 127.0), 32, -1)
    a = np.abs(x) / f
    assert a.max() <= 7.0
    half_step = np.where(a < 2, 0.25, np.where(a < 4, 0.5, 1.0))
    assert (np.abs(np.abs(y) / f - a) <= half_step).all()
    # a scale half as large would not hold the block
    assert (np.abs(x).reshape(200, 2, 32).max(-1) > 3.5 * 2.0 ** (scale - 127.0)).all()


@pytest.mark.parametrize("a,code", [(0.25, 0), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5.0, 6),
                                    (7.0, 7), (0.26, 1), (0.74, 1), (4.99, 6), (5.01, 7)])
def test_ties_go_to_the_even_code(a, code):
    x = np.zeros(32)
    x[0], x[1], x[2] = 6.5, a, -a  # the scale stays 1
    c, s = R.encode(x)
    assert s == 127 and c[1] == code and c[2] == code + 8


def test_extremes():
    x = np.zeros((5, 32))
    x[1, 3], x[2, 3], x[3, 3], x[4, 3] = np.inf, np.nan, 3.38e38, 1e-38
    y = R.round4(x)
    assert (y[0] == 0).all() and np.isnan(y[1:3]).all()
    assert np.isfinite(y[3]).all() and y[3, 3] == 6 * 2.0 ** 125
    assert y[4, 3] == 0  # below a quarter of the least scale


@pytest.mark.parametrize("d", [64, 128])
def test_places_cover_a_block_once(d):
    k, v, ks, vs = R.places(d)
    codes = np.concatenate((k[:, 0::2].ravel(), v[:, 0::2].ravel(), ks.ravel(), vs.ravel()))
    assert sorted(codes) == list(range(17 * d))
    assert (k[:, 0::2] == k[:, 1::2]).all() and (v[:, 0::2] == v[:, 1::2]).all()


def test_write_then_read():
    rng = np.random.default_rng(2)
    pool = rng.integers(0, 256, (3, 2, 17 * 64)).astype(np.uint8)
    before = [x.copy() for x in R.read_pool(pool, 64)]
    rows = R.bf16(rng.standard_normal((2, 2, 2, 64)))
    R.write_slots(pool, [0, 2], [5, 15], rows[0], rows[1])
    after = R.read_pool(pool, 64)
    for x, y, r in zip(before, after, rows):
        assert (y[0, :, 5] == R.round4(r[0])).all() and (y[2, :, 15] == R.round4(r[1])).all()
        y[0, :, 5], y[2, :, 15] = x[0, :, 5], x[2, :, 15]
        assert np.array_equal(x, y, equal_nan=True)


def test_mass_of_a_whole_row_is_its_heads():
    rng = np.random.default_rng(3)
    q, k = rng.standard_normal((5, 4, 8)), rng.standard_normal((12, 2, 8))
    _, lse, _, _ = R.attention(q, k, k, 7, 0.3)
    m = R.mass(q, lse, k, 7, 0.3)
    assert np.allclose(m.sum(0), 5 * 2)           # every (token, head) row spends 1
    assert not np.allclose(R.mass(q, lse + 0.01, k, 7, 0.3).sum(0), 10)
    assert (R.mass(q[:1], lse[:1], k, 7, 0.3)[8:] == 0).all()  # later keys are not seen


def test_kept_positions():
    s = np.array([3.0, 1.0, np.nan, 3.0, -np.inf, 2.0, 0.0, 9.0])
    assert list(R.kept(s, 3, 0)) == [0, 3, 7]
    assert list(R.kept(s, 3, 2)) == [0, 6, 7]      # the tie goes to the earlier
    assert list(R.kept(s, 7, 0)) == [0, 1, 3, 4, 5, 6, 7]
    assert list(R.kept(s, 8, 0)) == list(range(8))
    assert list(R.kept(s, 0, 0)) == []
