"""The 4-bit cache on the GPU: storing, reading back and the attention over it, against
tests/cache_reference.py in 64 bits."""
import numpy as np
import pytest
import torch

import cache_reference as R
import paper_2608_10402_amd as tide

pytestmark = pytest.mark.gpu

PAGE = 16


def rows_to_dev(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(torch.bfloat16).to("cuda")


def host(t):
    return t.double().cpu().numpy()


def make_table(rng, lens, extra=3):
    """Scattered pages for contexts of `lens`, and the number of pool pages."""
    n = [-(-int(x) // PAGE) for x in lens]
    pages = sum(n) + extra
    order = rng.permutation(pages)
    table = np.zeros((len(lens), max(max(n), 1)), np.int32)
    at = 0
    for b, k in enumerate(n):
        table[b, :k] = order[at:at + k]
        table[b, k:] = pages + 7  # never read
        at += k
    return table, pages


class Filled:
    """A pool whose first lens[b] positions per task hold random rows, with a host copy."""

    def __init__(self, seed, lens, hq, hkv, d, scale=1.0):
        self.rng = np.random.default_rng(seed)
        self.hq, self.hkv, self.d, self.lens = hq, hkv, d, np.asarray(lens, np.int32)
        table, pages = make_table(self.rng, lens)
        self.table = table
        self.kv = tide.PagedKV4(pages, hq, hkv, d, table)
        n = int(self.lens.sum())
        self.k, self.v = (R.bf16(self.rng.standard_normal((n, hkv, d)) * scale) for _ in range(2))
        self.kv.append(rows_to_dev(self.k), rows_to_dev(self.v), np.zeros(len(lens), np.int32), self.lens)
        self.k4, self.v4 = R.round4(self.k), R.round4(self.v)
        self.start = np.concatenate(([0], np.cumsum(self.lens)))

    def task(self, b, n=None):
        s = slice(self.start[b], self.start[b] + (self.lens[b] if n is None else n))
        return self.k4[s], self.v4[s]

    def queries(self, rows):
        return R.bf16(self.rng.standard_normal((rows, self.hq, self.d)))


def check(out, lse, ref):
    o, z, spread, size = ref
    assert np.isfinite(out).all()
    worst = (np.abs(out - o) - R.out_bound(o, spread)).max()
    assert worst <= 0, "output off by %g more than the bound" % worst
    if lse is not None:
        off = np.abs(lse - z).max()
        assert off <= R.score_bound(out.shape[-1], size) + 2.0 ** -22 * np.abs(z).max(), off


STORE = [  # prefix, extend, heads, d
    ([0], [1], 1, 64), ([15], [1], 2, 128), ([3, 0, 40], [5, 33, 0], 4, 128), ([7, 16, 31], [60, 16, 2], 5, 64),
    ([1000], [129], 3, 128), ([0] * 40, [17] * 40, 1, 128)]


@pytest.mark.parametrize("prefix,extend,hkv,d", STORE)
def test_append_stores_the_definition_and_nothing_else(prefix, extend, hkv, d):
    rng = np.random.default_rng(len(prefix) + d)
    total = np.array(prefix) + extend
    table, pages = make_table(rng, total)
    kv = tide.PagedKV4(pages, hkv, hkv, d, table)
    before = rng.integers(0, 256, tuple(kv.pool.shape), dtype=np.uint8)
    kv.pool.copy_(torch.from_numpy(before))
    n = int(np.sum(extend))
    k, v = (R.bf16(rng.standard_normal((n, hkv, d)) * np.exp2(rng.integers(-9, 9, (n, hkv, 1)))) for _ in range(2))
    k[rng.random(k.shape) < 0.02] *= 16  # outliers
    kv.append(rows_to_dev(k), rows_to_dev(v), prefix, extend)
    want = before.copy()
    pos = np.concatenate([np.arange(p, p + e) for p, e in zip(prefix, extend)])
    task = np.repeat(np.arange(len(prefix)), extend)
    R.write_slots(want, table[task, pos // PAGE], pos % PAGE, k, v)
    assert np.array_equal(kv.pool.cpu().numpy(), want)
    got_k, got_v = kv.unpack(prefix, extend)
    assert np.array_equal(host(got_k), R.round4(k)) and np.array_equal(host(got_v), R.round4(v))


@pytest.mark.parametrize("d", [64, 128])
def test_values_at_the_edges_of_the_format(d):
    """Zeros of both signs, subnormals, every tie, the largest values, NaN and infinities."""
    x = np.zeros((24, 1, d))
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0])
    for i, s in enumerate((-130, -126, -121, -120, -119, -20, 0, 1, 100, 121, 122, 123)):
        x[i, 0, 0:8] = ties * 2.0 ** s
        x[i, 0, 8:16] = -ties * 2.0 ** s
    x[12, 0, :] = -0.0
    x[13, 0, 5] = 2.0 ** -133
    x[14, 0, 7] = float.fromhex("0x1.fep127")
    x[15, 0, 9] = -float.fromhex("0x1.fep127")
    x[16, 0, 1], x[17, 0, 33], x[18, 0, d - 1] = np.nan, np.inf, -np.inf
    x[19, 0, :] = 1.0
    x = R.bf16(x)
    kv = tide.PagedKV4(2, 1, 1, d, [[1, 0]])
    kv.append(rows_to_dev(x), rows_to_dev(x[::-1]), [0], [24])
    k, v = kv.unpack([0], [24])
    assert np.array_equal(host(k), R.round4(x), equal_nan=True)
    assert np.array_equal(host(v), R.round4(x[::-1]), equal_nan=True)
    assert np.isnan(host(k)).sum() == 3 * 32


DECODE = [  # hq, hkv, d, lens
    (1, 1, 128, [1]), (8, 2, 64, [1, 2, 15, 16, 17, 31, 32, 33, 47, 48, 49]), (7, 1, 128, [100, 7, 1000]),
    (28, 4, 128, [300, 1999, 45]), (16, 1, 64, [513]), (16, 1, 128, [2048, 5]), (32, 8, 128, list(range(1, 130, 9))),
    (4, 4, 64, [4097]), (32, 2, 64, [6000]), (64, 8, 128, [777, 1]), (28, 4, 128, [40] * 70),
    (2500, 2500, 64, [70, 5]),                              # more kv heads than waves
    (8, 4, 64, [1 + 37 * i % 60 for i in range(1500)])]     # more tasks than runs


@pytest.mark.parametrize("hq,hkv,d,lens", DECODE)
def test_decode(hq, hkv, d, lens):
    f = Filled(hq * 1000 + d + len(lens), lens, hq, hkv, d)
    q = f.queries(len(lens))
    lse = torch.full((len(lens), hq), float("nan"), device="cuda")
    out = f.kv.decode(rows_to_dev(q), f.lens, lse=lse)
    again = f.kv.decode(rows_to_dev(q), f.lens)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16))
    for b in range(len(lens)):
        k, v = f.task(b)
        check(host(out)[b:b + 1], host(lse)[b:b + 1], R.attention(q[b:b + 1], k, v, lens[b] - 1, d ** -0.5))


@pytest.mark.parametrize("hq,hkv,d,lens", [(28, 4, 128, [300, 16, 1, 33, 32]), (8, 2, 64, [17, 1, 500, 64]),
                                           (16, 1, 128, [1500]), (5, 5, 64, list(range(1, 70)))])
def test_decode_append_is_append_then_decode(hq, hkv, d, lens):
    f = Filled(d + hq, lens, hq, hkv, d)
    n = len(lens)
    q, k, v = rows_to_dev(f.queries(n)), *(rows_to_dev(R.bf16(f.rng.standard_normal((n, hkv, d)))) for _ in range(2))
    pool = f.kv.pool.clone()
    lse = torch.empty((n, hq), device="cuda")
    out = f.kv.decode_append(q, k, v, f.lens, lse=lse)
    fused = f.kv.pool.clone()
    f.kv.pool.copy_(pool)
    f.kv.append(k, v, f.lens - 1, np.ones(n, np.int32))
    assert torch.equal(fused, f.kv.pool)
    lse2 = torch.empty_like(lse)
    assert torch.equal(out, f.kv.decode(q, f.lens, lse=lse2)) and torch.equal(lse, lse2)


EXTEND = [  # hq, hkv, d, prefix, extend
    (28, 4, 128, [37, 0, 200], [1, 2, 3]),            # few tokens: the codes themselves
    (32, 8, 128, [1000, 15, 16, 0], [8, 5, 0, 1]),
    (16, 1, 64, [300], [7]), (3, 3, 64, [64, 1], [16, 16]), (1, 1, 128, [5], [16]),
    (16, 1, 128, [64, 7], [2, 1]), (28, 4, 128, [300, 33], [48, 2]), (32, 2, 64, [500, 70], [12, 5]),  # several units
    (28, 4, 128, [100, 0, 411], [130, 17, 1]),        # staged
    (8, 2, 64, [37, 250, 0], [5, 0, 200]), (16, 1, 128, [0], [65]), (4, 4, 128, [90], [300])]


@pytest.mark.parametrize("hq,hkv,d,prefix,extend", EXTEND)
def test_extend(hq, hkv, d, prefix, extend):
    total = np.array(prefix) + extend
    f = Filled(d + sum(extend), total, hq, hkv, d)
    rows = int(np.sum(extend))
    q = f.queries(rows)
    lse = torch.full((rows, hq), float("nan"), device="cuda")
    out = f.kv.extend(rows_to_dev(q), prefix, extend, lse=lse)
    at = 0
    for b, (p, e) in enumerate(zip(prefix, extend)):
        if e == 0:
            continue
        k, v = f.task(b)
        check(host(out)[at:at + e], host(lse)[at:at + e], R.attention(q[at:at + e], k, v, p, d ** -0.5))
        at += e


def test_extend_rows_outside_the_call_stay():
    f = Filled(5, [60, 40], 8, 2, 64)
    for extend in ([4, 3], [4, 30]):
        rows = sum(extend)
        q = rows_to_dev(f.queries(rows))
        buf = torch.full((rows + 4, 8, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        f.kv.extend(q, f.lens - np.array(extend, np.int32), extend, out=buf[2:2 + rows])
        assert (buf[:2] == 7).all() and (buf[2 + rows:] == 7).all() and not (buf[2:2 + rows] == 7).all()


def test_large_scores_and_single_winner():
    """Scores far apart: one key takes all the weight, far into the context."""
    f = Filled(11, [700], 8, 2, 128)
    k, v = f.task(0)
    q = np.repeat(k[650].reshape(1, 2, 1, 128), 4, 2).reshape(1, 8, 128) * 30
    q = R.bf16(q)
    out = f.kv.decode(rows_to_dev(q), [700])
    check(host(out), None, R.attention(q, k, v, 699, 128 ** -0.5))


@pytest.mark.parametrize("call", ["decode", "extend_few", "extend", "append", "unpack", "decode_append"])
def test_bad_page_ids_are_reported_and_never_read(call, monkeypatch):
    f = Filled(3, [100, 60], 8, 2, 64)
    good = f.kv.pool.clone()
    bad = f.table.copy()
    bad[0, 2], bad[1, 3] = -5, 1 << 30
    bad[1, 4:] = 0
    f.kv.set_block_table(bad)
    new = [rows_to_dev(f.queries(160)[:, :2]) for _ in range(2)]
    q = rows_to_dev(f.queries(160))

    def go():
        if call == "decode":
            return f.kv.decode(q[:2], f.lens)
        if call == "decode_append":
            return f.kv.decode_append(q[:2], new[0][:2], new[1][:2], f.lens)
        if call == "extend_few":
            return f.kv.extend(q[:4], f.lens - 2, [2, 2])
        if call == "extend":
            return f.kv.extend(q[:140], f.lens - np.array([90, 50], np.int32), [90, 50])  # (unpacked pages)
        if call == "append":
            return f.kv.append(*new, [0, 0], f.lens)
        return f.kv.unpack([0, 0], f.lens)

    got = go()
    torch.cuda.synchronize()
    if call == "unpack":
        assert (got[0][32:48] == 0).all() and (got[1][100 + 48:] == 0).all()
    if call == "append":  # every other slot of the two tasks is written
        want = good.cpu().numpy()
        pos = np.concatenate((np.arange(100), np.arange(60)))
        page = bad[np.repeat([0, 1], [100, 60]), pos // PAGE]
        ok = (page >= 0) & (page < f.kv.num_pages)
        R.write_slots(want, page[ok], (pos % PAGE)[ok], host(new[0])[ok], host(new[1])[ok])
        assert np.array_equal(f.kv.pool.cpu().numpy(), want)
    monkeypatch.setenv("TIDE_DEBUG_CHECKS", "1")
    with pytest.raises(tide.TideError) as e:
        go()
    assert e.value.status == tide.TIDE_ERR_PAGE_RANGE


def test_result_does_not_depend_on_the_pages():
    a = Filled(21, [513, 90], 28, 4, 128)
    q = rows_to_dev(a.queries(2))
    one = a.kv.decode(q, a.lens)
    perm = np.random.default_rng(9).permutation(a.kv.num_pages)
    inverse = np.argsort(perm)
    moved = a.table.copy()
    ok = moved < a.kv.num_pages
    moved[ok] = inverse[moved[ok]]
    b = tide.PagedKV4(a.kv.num_pages, 28, 4, 128, moved, pool=a.kv.pool[torch.from_numpy(perm).cuda()].contiguous())
    assert torch.equal(one, b.decode(q, a.lens))


def test_offsets_past_32_bits():
    """Pages beyond 4 GiB of the pool."""
    pages = (5 << 30) // (8 * 17 * 128)
    table = np.array([[pages - 1, 3, pages - 2]], np.int32)
    kv = tide.PagedKV4(pages, 32, 8, 128, table, fill_canary=False)
    rng = np.random.default_rng(4)
    k, v = (R.bf16(rng.standard_normal((40, 8, 128))) for _ in range(2))
    kv.append(rows_to_dev(k), rows_to_dev(v), [0], [40])
    k4, v4 = R.round4(k), R.round4(v)
    got = kv.unpack([0], [40])
    assert np.array_equal(host(got[0]), k4) and np.array_equal(host(got[1]), v4)
    q = R.bf16(rng.standard_normal((20, 32, 128)))
    for e in (1, 2, 20):
        out = kv.extend(rows_to_dev(q[:e]), [40 - e], [e])
        check(host(out), None, R.attention(q[:e], k4, v4, 40 - e, 128 ** -0.5))
    out = kv.decode(rows_to_dev(q[:1]), [40])
    check(host(out), None, R.attention(q[:1], k4, v4, 39, 128 ** -0.5))


@pytest.mark.parametrize("unpacked", [False, True])
def test_other_stream_and_graph_replays(unpacked):
    """Captured calls, replayed between eager ones on other data, against the eager results."""
    f = Filled(31, [200, 77, 1], 28, 4, 128)
    n = 3
    q, k, v = rows_to_dev(f.queries(n)), *(rows_to_dev(R.bf16(f.rng.standard_normal((n, 4, 128)))) for _ in range(2))
    new = [150, 70, 0] if unpacked else [40, 30, 0]
    qx = rows_to_dev(f.queries(sum(new)))
    ext = (f.lens - np.array(new, np.int32), new)
    info = tide.tide_plan_info_get(tide.TIDE_OP_KV4_EXTEND, *ext, f.kv.dims)
    assert (info["run_steps"] == 0) == unpacked
    pool = f.kv.pool.clone()
    want = f.kv.decode_append(q, k, v, f.lens).clone()
    wantx = f.kv.extend(qx, *ext).clone()
    want_pool = f.kv.pool.clone()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        side.wait_stream(torch.cuda.default_stream())
        assert torch.equal(f.kv.decode(q, f.lens), want)
    torch.cuda.synchronize()
    out, outx = torch.empty_like(want), torch.empty_like(wantx)
    kv2 = tide.PagedKV4(f.kv.num_pages, 28, 4, 128, f.table, pool=f.kv.pool)  # a workspace of the graph's own
    kv2.workspace(tide.tide_workspace_size(tide.TIDE_OP_KV4_EXTEND, *ext, kv2.dims))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        kv2.decode_append(q, k, v, f.lens, out=out)
        kv2.extend(qx, *ext, out=outx)
    for i in range(20):
        f.kv.pool.copy_(pool)
        out.zero_()
        outx.zero_()
        f.kv.decode(q, f.lens)
        g.replay()
        assert torch.equal(out, want) and torch.equal(outx, wantx) and torch.equal(f.kv.pool, want_pool), i
