"""Attention mass and eviction on the GPU, over the bf16 and the 4-bit cache, against
tests/cache_reference.py; and the operators in a row, as a rollout engine calls them."""
import numpy as np
import pytest
import torch

import cache_reference as R
import paper_2608_10402_amd as tide
from test_gpu_kv4 import PAGE, host, make_table, rows_to_dev

pytestmark = pytest.mark.gpu


class Cache:
    """A pool of either kind with random contexts and random sums, and host copies of both."""

    def __init__(self, seed, lens, hq, hkv, d, bits, extra=3):
        self.rng = np.random.default_rng(seed)
        self.hq, self.hkv, self.d, self.bits, self.lens = hq, hkv, d, bits, np.asarray(lens, np.int32)
        self.table, pages = make_table(self.rng, lens, extra)
        cls = tide.PagedKV4 if bits == 4 else tide.PagedKV
        self.kv = cls(pages, hq, hkv, d, self.table)
        n = int(self.lens.sum())
        k, v = (R.bf16(self.rng.standard_normal((n, hkv, d))) for _ in range(2))
        if n:
            self.kv.append(rows_to_dev(k), rows_to_dev(v), np.zeros(len(lens), np.int32), self.lens)
        self.k, self.v = (R.round4(k), R.round4(v)) if bits == 4 else (k, v)
        self.sums = np.exp(2 * self.rng.standard_normal((pages, hkv, PAGE))).astype(np.float32)
        self.start = np.concatenate(([0], np.cumsum(self.lens)))

    def mass(self):
        return torch.from_numpy(self.sums.copy()).cuda()

    def rows(self, b):
        s = slice(self.start[b], self.start[b + 1])
        return self.k[s], self.v[s]

    def read(self):
        """K and V of every slot [pages][Hkv][16][d]."""
        if self.bits == 4:
            return R.read_pool(self.kv.pool.cpu().numpy(), self.d)
        return host(self.kv.k_pool), host(self.kv.v_pool)


MASS = [  # hq, hkv, d, prefix, extend
    (1, 1, 128, [0], [1]), (28, 4, 128, [200, 15, 16], [1, 1, 1]), (8, 2, 64, [0, 63, 64, 300], [1, 2, 65, 0]),
    (16, 1, 64, [511], [3]), (5, 5, 128, [100], [40]), (28, 4, 128, [1000, 5], [33, 90]), (32, 2, 64, [0], [300])]


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("hq,hkv,d,prefix,extend", MASS)
@pytest.mark.parametrize("counted", [None, "none", "some"])
def test_mass(hq, hkv, d, prefix, extend, counted, bits):
    total = np.array(prefix) + extend
    c = Cache(d + sum(extend), total, hq, hkv, d, bits)
    q = R.bf16(c.rng.standard_normal((int(np.sum(extend)), hq, d)))
    scale = d ** -0.5
    lens = {None: None, "none": np.zeros(len(prefix), np.int32), "some": total // 2}[counted]
    carried = prefix if lens is None else lens
    mass = c.mass()
    lse, want, bound, at = np.zeros((len(q), hq)), c.sums.astype(np.float64), np.zeros(c.sums.shape), 0
    for b, (p, e) in enumerate(zip(prefix, extend)):
        if e == 0:
            continue
        k, v = c.rows(b)
        _, z, _, size = R.attention(q[at:at + e], k, v, p, scale)
        lse[at:at + e] = z.astype(np.float32)
        got = R.mass(q[at:at + e], lse[at:at + e], k, p, scale)
        pos = np.arange(p + e)
        page, slot = c.table[b][pos // PAGE], pos % PAGE
        old = np.where(pos < carried[b], want[page, :, slot].T, 0.0).T
        want[page, :, slot] = old + got
        # each weight: the score's error, and the log-sum-exp's conversion to base 2 and the exponential's
        # own; the sum: one rounding an addend
        rel = 2 * R.score_bound(d, size) + 2.0 ** -22 * np.abs(z).max() + 2.0 ** -21
        rounds = 2.0 ** -24 * (e * hq // hkv + 20)
        bound[page, :, slot] = got * (rel + rounds) + 2.0 ** -24 * (old + got) + 1e-38
        at += e
    c.kv.attn_mass(rows_to_dev(q), torch.from_numpy(lse.astype(np.float32)).cuda(), prefix, extend, mass,
                   counted_lens=lens)
    off = np.abs(host(mass) - want) - bound
    assert off.max() <= 0, (off.max(), np.unravel_index(off.argmax(), off.shape))
    again = c.mass()
    c.kv.attn_mass(rows_to_dev(q), torch.from_numpy(lse.astype(np.float32)).cuda(), prefix, extend, again,
                   counted_lens=lens)
    assert torch.equal(mass, again)


@pytest.mark.parametrize("bits", [16, 4])
def test_mass_ignores_what_lies_past_the_context(bits):
    """Unused slots hold NaN (the pools' canary); with the rows' own log-sum-exps every row spends
    1 on the context's keys."""
    c = Cache(8, [37, 70], 8, 2, 128, bits)
    q = rows_to_dev(c.rng.standard_normal((5, 8, 128)))
    lse = torch.empty((5, 8), device="cuda")
    prefix, extend = np.array([35, 67], np.int32), [2, 3]
    c.kv.extend(q, prefix, extend, lse=lse)
    mass = c.kv.new_mass()
    c.kv.attn_mass(q, lse, prefix, extend, mass)
    m = host(mass)
    assert np.isfinite(m).all()
    for b, e in enumerate(extend):
        mine = m[c.table[b, : -(-c.lens[b] // PAGE)]]
        assert np.abs(mine.sum((0, 2)) - e * 4).max() < 1e-4  # 12 rows of weights, each 1 within 1e-5


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("prefix,extend,bad", [(35, 5, 2), (61, 9, 3), (70, 30, 7), (0, 1, 0)])
def test_mass_of_rows_that_are_not_numbers(prefix, extend, bad, bits):
    """A row whose log-sum-exp is NaN or -inf reaches the keys that it sees, of its kv head, and no other; a
    key that scores -inf with every row gets nothing."""
    c = Cache(extend, [prefix + extend], 12, 2, 64, bits)
    q = np.abs(c.rng.standard_normal((extend, 12, 64))) + 2.0 ** -6
    lse = np.full((extend, 12), 4.0, np.float32)
    lost = prefix + extend - 1  # (a key of the 4-bit cache holds no infinity)
    if bits == 16:
        c.kv.k_pool[int(c.table[0, lost // PAGE]), 1, lost % PAGE] = -np.inf
    want = c.kv.new_mass()
    c.kv.attn_mass(rows_to_dev(q), torch.from_numpy(lse).cuda(), [prefix], [extend], want)
    pos = np.arange(prefix + extend)
    page, slot = c.table[0][pos // PAGE], pos % PAGE
    want = host(want)[page, :, slot]
    assert np.isfinite(want).all()
    if bits == 16:
        assert want[lost, 1] == 0 and want[lost, 0] > 0
    for value in (np.nan, -np.inf):
        lse[bad, :6] = value  # kv head 0
        mass = c.kv.new_mass()
        c.kv.attn_mass(rows_to_dev(q), torch.from_numpy(lse).cuda(), [prefix], [extend], mass)
        got = host(mass)[page, :, slot]
        reached = pos <= prefix + bad
        assert not np.isfinite(got[reached, 0]).any()
        assert np.array_equal(got[~reached, 0], want[~reached, 0]) and np.array_equal(got[:, 1], want[:, 1])


def check_evict(c, mass0, keep, recent, new_table=None, give_kept=True):
    """Evicts and compares pools, sums and kept positions with the definition, every slot."""
    mass = torch.from_numpy(mass0.copy()).cuda()
    k0, v0 = (x.copy() for x in c.read())
    total = int(np.sum(keep))
    new = None if new_table is None else torch.from_numpy(new_table).cuda()
    kept = torch.full((total, c.hkv), -1, dtype=torch.int32, device="cuda") if give_kept else None
    got = c.kv.evict(mass, c.lens, keep, recent_lens=recent, new_block_table=new, kept=kept)
    k1, v1 = c.read()
    m1 = mass.cpu().numpy()
    to = c.table if new_table is None else new_table
    want_k, want_v, want_m, at = k0.copy(), v0.copy(), mass0.copy(), 0
    for b, n in enumerate(c.lens):
        pos = np.arange(n)
        page, slot = c.table[b][pos // PAGE], pos % PAGE
        r = np.arange(keep[b])
        tp, ts = to[b][r // PAGE], r % PAGE
        for h in range(c.hkv):
            idx = R.kept(mass0[page, h, slot], keep[b], 0 if recent is None else recent[b])
            assert np.array_equal(got[at:at + keep[b], h].cpu().numpy(), idx), (b, h)
            for want, old in ((want_k, k0), (want_v, v0), (want_m, mass0)):
                want[tp, h, ts] = old[page[idx], h, slot[idx]]
        at += keep[b]
    assert np.array_equal(m1, want_m, equal_nan=True)
    assert np.array_equal(k1, want_k, equal_nan=True) and np.array_equal(v1, want_v, equal_nan=True)


EVICT = [  # hkv, d, lens, keep, recent
    (1, 128, [1], [1], [0]), (2, 64, [40, 17, 16], [20, 17, 1], [5, 0, 1]), (4, 128, [333, 100], [100, 0], [16, 0]),
    (1, 64, [5000], [1234], [100]), (3, 128, [2100, 1, 900], [2099, 1, 450], [0, 1, 450]), (2, 128, [64, 0], [63, 0], None),
    (1, 128, [9001], [8200], [1]), (2, 64, [700] * 9, [300] * 9, [32] * 9)]


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("inplace", [True, False])
@pytest.mark.parametrize("hkv,d,lens,keep,recent", EVICT)
def test_evict(hkv, d, lens, keep, recent, inplace, bits):
    room = 0 if inplace else sum(-(-k // PAGE) for k in keep)
    c = Cache(len(lens) + d, lens, hkv * 2, hkv, d, bits, extra=3 + room)
    new = None
    if not inplace:
        free = [p for p in range(c.sums.shape[0]) if p not in set(c.table.ravel())]
        c.rng.shuffle(free)
        new = np.full((len(lens), max(1, max(-(-k // PAGE) for k in keep))), 1 << 20, np.int32)
        for b, k in enumerate(keep):
            for i in range(-(-k // PAGE)):
                new[b, i] = free.pop()
    check_evict(c, c.sums, keep, recent, new)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("kind", ["equal", "two", "nan", "zeros", "inf", "negative", "tiny"])
def test_evict_ties_and_odd_sums(kind, bits):
    c = Cache(77, [1000, 50], 4, 2, 64, bits)
    m = c.sums.copy()
    pick = c.rng.random(m.shape)
    if kind == "equal":
        m[:] = 0.125
    elif kind == "two":
        m[:] = np.where(pick < 0.5, 1.0, 2.0)
    elif kind == "nan":
        m[pick < 0.7] = np.nan
        m[(pick > 0.7) & (pick < 0.75)] = -np.inf
    elif kind == "zeros":
        m[:] = np.where(pick < 0.5, 0.0, -0.0)
    elif kind == "inf":
        m[pick < 0.3] = np.inf
    elif kind == "negative":
        m *= np.where(pick < 0.5, -1, 1)
    else:
        m[:] = (pick * 50).astype(np.int32) * np.float32(1e-45)
    check_evict(c, m, [400, 25], [10, 0])


def test_evict_leaves_what_a_bad_page_holds(monkeypatch):
    c = Cache(5, [100, 60], 4, 2, 64, 16)
    bad = c.table.copy()
    bad[0, 1] = -1
    c.kv.set_block_table(bad)
    mass = c.mass()
    before = c.read()[0].copy()
    c.kv.evict(mass, c.lens, [50, 30])
    torch.cuda.synchronize()
    after = c.read()[0]
    others = [p for p in range(len(before)) if p not in set(c.table[0, :4]) | set(c.table[1, :2])]
    assert np.array_equal(before[others], after[others], equal_nan=True)
    monkeypatch.setenv("TIDE_DEBUG_CHECKS", "1")
    for call in (lambda: c.kv.evict(mass, c.lens, [50, 30]),
                 lambda: c.kv.attn_mass(torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda"),
                                        torch.zeros((2, 4), device="cuda"), c.lens - 1, [1, 1], mass)):
        with pytest.raises(tide.TideError) as e:
            call()
        assert e.value.status == tide.TIDE_ERR_PAGE_RANGE


def test_shared_source_pages_into_pages_of_their_own():
    """Two trajectories of a group share their prompt's pages; each keeps its own choice of them."""
    c = Cache(13, [160], 4, 2, 128, 16, extra=20)
    free = [p for p in range(c.sums.shape[0]) if p not in set(c.table.ravel())]
    table = np.concatenate((c.table, c.table))
    new = np.array([free[:5], free[5:10]], np.int32)
    c.kv.set_block_table(table)
    mass = c.mass()
    kept = c.kv.evict(mass, [160, 150], [80, 75], recent_lens=[8, 8], new_block_table=torch.from_numpy(new).cuda())
    k = c.read()[0]
    for b, (n, m, at) in enumerate(((160, 80, 0), (150, 75, 80))):
        pos = np.arange(n)
        for h in range(2):
            idx = R.kept(c.sums[table[b][pos // PAGE], h, pos % PAGE], m, 8)
            assert np.array_equal(kept[at:at + m, h].cpu().numpy(), idx)
            r = np.arange(m)
            assert np.array_equal(k[new[b][r // PAGE], h, r % PAGE], c.rows(0)[0][idx, h])


@pytest.mark.parametrize("bits", [16, 4])
def test_pools_past_32_bits(bits):
    """Pages beyond 4 GiB of the pools."""
    hkv, d = 8, 128
    pages = (9 << 29) // (hkv * (17 * d if bits == 4 else 2 * PAGE * d))
    table = np.array([[pages - 1, pages - 3, 2]], np.int32)
    kv = (tide.PagedKV4 if bits == 4 else tide.PagedKV)(pages, 32, hkv, d, table, fill_canary=False)
    rng = np.random.default_rng(3)
    k, v = (R.bf16(rng.standard_normal((48, hkv, d))) for _ in range(2))
    kv.append(rows_to_dev(k), rows_to_dev(v), [0], [48])
    q = rows_to_dev(rng.standard_normal((1, 32, d)))
    lse = torch.empty((1, 32), device="cuda")
    kv.decode(q, [48], lse=lse)
    mass = kv.new_mass()
    kv.attn_mass(q, lse, [47], [1], mass)
    m = host(mass[torch.from_numpy(table[0]).long().cuda()]).transpose(0, 2, 1).reshape(48, hkv)
    assert np.abs(m.sum(0) - 4).max() < 1e-4
    kept = kv.evict(mass, [48], [20]).cpu().numpy()
    back = kv.unpack([0], [20])[0] if bits == 4 else None
    for h in range(hkv):
        assert np.array_equal(kept[:, h], R.kept(m[:, h], 20, 0))
        want = (R.round4(k) if bits == 4 else k)[kept[:, h], h]
        got = host(back)[:, h] if bits == 4 else np.concatenate([host(kv.k_pool[p, h]) for p in table[0]])[:20]
        assert np.array_equal(got, want)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("hq,hkv,d", [(28, 4, 128), (8, 2, 64)])
def test_a_resumed_task_goes_on_after_eviction(hq, hkv, d, bits):
    """Prompt, scored by its last tokens, cut, extended, decoded token by token with sums carried
    on, cut again: attention at the end equals that over exactly the positions kept."""
    rng = np.random.default_rng(hq + bits)
    lens = np.array([300, 90], np.int32)
    table, pages = make_table(rng, lens + 64)
    kv = (tide.PagedKV4 if bits == 4 else tide.PagedKV)(pages, hq, hkv, d, table)
    mass = kv.new_mass()
    hist = [[] for _ in lens]  # rows (k, v) as stored, per task, in cache order per head
    stored = R.round4 if bits == 4 else (lambda x: x)

    def fresh(extend):
        n = int(np.sum(extend))
        k, v = (R.bf16(rng.standard_normal((n, hkv, d))) for _ in range(2))
        at = 0
        for b, e in enumerate(extend):
            hist[b].extend(zip(stored(k)[at:at + e], stored(v)[at:at + e]))
            at += e
        return k, v, R.bf16(rng.standard_normal((n, hq, d)))

    def cut(now, keep, recent):
        kept = kv.evict(mass, now, keep, recent_lens=recent).cpu().numpy()
        at = 0
        for b, m in enumerate(keep):
            k, v = (np.stack([r[i] for r in hist[b]]) for i in range(2))
            idx = kept[at:at + m]
            assert (np.diff(idx, axis=0) > 0).all() and (idx[m - recent[b]:] >= now[b] - recent[b]).all()
            k, v = (np.stack([x[idx[:, h], h] for h in range(hkv)], 1) for x in (k, v))
            hist[b] = list(zip(k, v))
            at += m
        return np.asarray(keep, np.int32)

    def attend(q, prefix, extend, out, lse):
        at = 0
        for b, (p, e) in enumerate(zip(prefix, extend)):
            k, v = (np.stack([r[i] for r in hist[b]]) for i in range(2))
            o, z, spread, size = R.attention(q[at:at + e], k, v, p, d ** -0.5)
            assert (np.abs(host(out)[at:at + e] - o) <= R.out_bound(o, spread)).all()
            assert np.abs(host(lse)[at:at + e] - z).max() <= R.score_bound(d, size) + 2.0 ** -22 * np.abs(z).max()
            at += e

    k, v, q = fresh(lens)
    kv.append(rows_to_dev(k), rows_to_dev(v), [0, 0], lens)
    lse = torch.empty((int(lens.sum()), hq), device="cuda")
    (kv.extend(rows_to_dev(q), [0, 0], lens, lse=lse))
    w = np.array([16, 16], np.int32)  # the last tokens vote
    sel = np.concatenate((np.arange(300 - 16, 300), np.arange(390 - 16, 390)))
    kv.attn_mass(rows_to_dev(q[sel]), lse[torch.from_numpy(sel).cuda()].contiguous(), lens - w, w, mass,
                 counted_lens=[0, 0])
    now = cut(lens, [120, 50], [16, 8])
    new = [40, 21]
    k, v, q = fresh(new)
    kv.append(rows_to_dev(k), rows_to_dev(v), now, new)
    lse = torch.empty((61, hq), device="cuda")
    out = kv.extend(rows_to_dev(q), now, new, lse=lse)
    attend(q, now, new, out, lse)
    kv.attn_mass(rows_to_dev(q), lse, now, new, mass)
    now = now + new
    for _ in range(3):
        k, v, q = fresh([1, 1])
        now = now + 1
        lse = torch.empty((2, hq), device="cuda")
        out = kv.decode_append(rows_to_dev(q), rows_to_dev(k), rows_to_dev(v), now.astype(np.int32), lse=lse)
        attend(q, now - 1, [1, 1], out, lse)
        kv.attn_mass(rows_to_dev(q), lse, now - 1, [1, 1], mass)
    now = cut(now.astype(np.int32), [60, 60], [3, 3])
    k, v, q = fresh([1, 1])
    lse = torch.empty((2, hq), device="cuda")
    out = kv.decode_append(rows_to_dev(q), rows_to_dev(k), rows_to_dev(v), now + 1, lse=lse)
    attend(q, now, [1, 1], out, lse)


def test_graph_replays():
    """A captured step (sums, then an eviction into new pages), replayed between eager calls."""
    c = Cache(41, [200, 120], 8, 2, 128, 4, extra=30)
    free = np.array([p for p in range(c.sums.shape[0]) if p not in set(c.table.ravel())], np.int32)
    new = torch.from_numpy(free[:16].reshape(2, 8)).cuda()
    q = rows_to_dev(c.rng.standard_normal((2, 8, 128)))
    lse = torch.empty((2, 8), device="cuda")
    c.kv.decode(q, c.lens, lse=lse)
    pool = c.kv.pool.clone()

    def step(kv, mass, kept):
        kv.attn_mass(q, lse, c.lens - 1, [1, 1], mass)
        kv.evict(mass, c.lens, [100, 60], recent_lens=[8, 8], new_block_table=new, kept=kept)

    want_mass, want_kept = c.mass(), torch.empty((160, 2), dtype=torch.int32, device="cuda")
    step(c.kv, want_mass, want_kept)
    want_pool = c.kv.pool.clone()
    kv2 = tide.PagedKV4(c.kv.num_pages, 8, 2, 128, c.table, pool=c.kv.pool)
    kv2.workspace(1 << 20)
    mass, kept = c.mass(), torch.empty_like(want_kept)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(kv2, mass, kept)
    for i in range(20):
        c.kv.pool.copy_(pool)
        mass.copy_(torch.from_numpy(c.sums))
        kept.zero_()
        c.kv.decode(q, c.lens, lse=lse)
        g.replay()
        assert torch.equal(mass, want_mass) and torch.equal(kept, want_kept) and torch.equal(c.kv.pool, want_pool), i


@pytest.mark.parametrize("bits", [16, 4])
def test_calls_on_two_streams_at_once(bits):
    """Two caches, each with a workspace and a stream of its own, in turn and without waits between."""
    caches = [Cache(7 + i, [400 + 90 * i, 33, 128], 16, 4, 128, bits) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in caches]
    qs = [rows_to_dev(c.rng.standard_normal((3, 16, 128))) for c in caches]
    keep = np.array([200, 20, 128], np.int32)

    def step(c, q, mass):
        """Decode, sums, eviction; returns what they wrote."""
        lse = torch.empty((3, 16), device="cuda")
        out = c.kv.decode(q, c.lens, lse=lse)
        c.kv.attn_mass(q, lse, c.lens - 1, [1, 1, 1], mass)
        return out, lse, mass.clone(), c.kv.evict(mass, c.lens, keep, recent_lens=[4, 4, 4])

    def pools(c):
        return [c.kv.pool] if bits == 4 else [c.kv.k_pool, c.kv.v_pool]

    start = [[p.clone() for p in pools(c)] for c in caches]
    want = [step(c, q, c.mass()) + tuple(p.clone() for p in pools(c)) for c, q in zip(caches, qs)]
    for turn in range(10):
        for c, p in zip(caches, start):
            for a, b in zip(pools(c), p):
                a.copy_(b)
        sums = [c.mass() for c in caches]
        torch.cuda.synchronize()
        got = []
        for c, q, m, s in zip(caches, qs, sums, streams):
            with torch.cuda.stream(s):
                got.append(step(c, q, m))
        torch.cuda.synchronize()
        for c, g, w in zip(caches, got, want):
            for x, y in zip(g + tuple(pools(c)), w):
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), turn
