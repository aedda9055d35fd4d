"""Page maps, key bounds, the choice of blocks and attention over them on the CPU, one element after the
other from the definitions in include/tide.h, in whole numbers or 64 bits; shared by the GPU tests."""
import numpy as np

PAGE = 16
LEAST, MOST, NONE = -120, 122, 127


def pages_of(n):
    return -(-int(n) // PAGE)


def page_map(lens, want, table, free, count, num_rows):
    """lens_out, table, free, count_out, row_start, rows [num_rows][3] (task, position, slot)."""
    table, free = np.array(table, np.int64), np.array(free, np.int64)
    lens, want = [int(x) for x in lens], [int(x) for x in want]
    n, most = len(lens), table.shape[1] * PAGE
    ok = [0 <= a <= most and 0 <= w <= most for a, w in zip(lens, want)]
    out, top = list(lens), min(max(int(count), 0), free.size)
    back = []
    for b in range(n):
        if ok[b] and want[b] < lens[b]:
            back += [table[b, i] for i in range(pages_of(want[b]), pages_of(lens[b]))]
            out[b] = want[b]
    for p in back:
        if top < free.size:
            free[top] = p
            top += 1
    rows, row_start, asked, needed, there = [], [], 0, 0, top
    for b in range(n):
        row_start.append(len(rows))
        if not ok[b] or want[b] <= lens[b]:
            continue
        asked += want[b] - lens[b]
        if asked > num_rows:
            continue
        first, end = pages_of(lens[b]), pages_of(want[b])
        needed += end - first
        if end > first and needed > there:
            rows += [(-1, -1, -1)] * (want[b] - lens[b])
            continue
        for i in range(first, end):
            top -= 1
            table[b, i] = free[top]
        out[b] = want[b]
        for p in range(lens[b], want[b]):
            page = table[b, p // PAGE]
            rows.append((b, p, -1 if page < 0 else page * PAGE + p % PAGE))
    row_start.append(len(rows))
    rows += [(-1, -1, -1)] * (num_rows - len(rows))
    return out, table, free, top, row_start, np.array(rows, np.int64).reshape(-1, 3)


def unit_of(top):
    """The least s in [-120, 122] with top <= 127 * 2^s, by trying them."""
    for s in range(LEAST, MOST):
        if top <= 127.0 * 2.0 ** s:
            return s
    return MOST


def bounds_of(k):
    """k [n][d]: (upper [d], lower [d], unit)."""
    k = np.asarray(k, np.float64)
    if not np.isfinite(k).all():
        return np.zeros(k.shape[1], np.int64), np.zeros(k.shape[1], np.int64), NONE
    s = unit_of(np.abs(k).max())
    return (np.ceil(k.max(0) / 2.0 ** s).astype(np.int64), np.floor(k.min(0) / 2.0 ** s).astype(np.int64), s)


def codes_of(q):
    """q [G][d] -> whole numbers [G][d] and their units [G]; zeros where a head is not finite."""
    code, unit = np.zeros(q.shape, np.int64), np.zeros(len(q), np.int64)
    for h in range(len(q)):
        if np.isfinite(q[h]).all():
            unit[h] = unit_of(np.abs(q[h]).max())
            code[h] = np.rint(q[h] / 2.0 ** unit[h])  # ties to even
    return code, unit


def scores(q, upper, lower, units):
    """q [G][d] (64 bits), bounds [blocks][d] -> [blocks], exact."""
    code, t = codes_of(q)
    out = np.full(len(units), -np.inf)
    for c, e in zip(code, t):
        whole = np.maximum(c * upper.astype(np.int64), c * lower.astype(np.int64)).sum(1)
        out = np.maximum(out, whole * 2.0 ** np.clip(units.astype(np.int64) + e, -100, 100))
    return np.where(units == NONE, np.inf, out)


def choose(score, blocks, budget, sink, recent):
    """Of the first `blocks` entries of score: `budget` indices, ascending, -1 behind them."""
    if blocks <= budget:
        pick = list(range(blocks))
    else:
        best = [sink + int(i) for i in np.argsort(-np.asarray(score[sink: blocks - recent]), kind="stable")]
        best = best[: budget - sink - recent]
        pick = list(range(sink)) + sorted(best) + list(range(blocks - recent, blocks))
    return pick + [-1] * (budget - len(pick))


def attend(q, k, v, blocks, pos, scale):
    """q [G][d] over the positions <= pos of the listed blocks; k, v [positions][d].  out, lse, sum of
    weight |v|, largest sum |q k| scale; zeros and -inf where nothing is listed."""
    at = [p for b in blocks if b >= 0 for p in range(PAGE * b, min(PAGE * (b + 1), pos + 1))]
    if not at:
        return np.zeros(q.shape), np.full(len(q), -np.inf), np.zeros(q.shape), 0.0
    k, v = k[at], v[at]
    s = q @ k.T * scale
    m = s.max(1, keepdims=True)
    p = np.exp(s - m)
    l = p.sum(1, keepdims=True)
    p = p / l
    return p @ v, (m + np.log(l))[:, 0], p @ np.abs(v), (np.abs(q) @ np.abs(k).T).max() * scale
