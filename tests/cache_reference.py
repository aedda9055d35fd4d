"""The 4-bit cache, attention mass and eviction in 64 bits on the CPU, from the definitions in
include/tide.h, entry by entry; shared by the GPU tests."""
import numpy as np

PAGE = 16
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def bf16(x):
    """float array -> the nearest bf16 values (ties to even), as float64."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32)
    return r.view(np.float32).astype(np.float64)


def encode(x):
    """Codes (0..15) [..., d] and scale bytes [..., d / 32] of rows x, by search over the grid."""
    b = np.asarray(x, np.float64)
    b = b.reshape(b.shape[:-1] + (-1, 32))
    finite = np.isfinite(b).all(-1)
    z = np.where(finite[..., None], b, 0.0)
    amax = np.abs(z).max(-1)
    s = np.full(amax.shape, 125)
    for e in range(125, -121, -1):  # the least exponent that holds the block
        s = np.where(amax <= 7.0 * 2.0 ** e, e, s)
    a = np.abs(z) / (2.0 ** s.astype(np.float64))[..., None]
    dist = np.abs(a[..., None] - GRID)
    near = dist == dist.min(-1, keepdims=True)
    two = near.sum(-1, keepdims=True) == 2
    code = np.where(two, near & (np.arange(8) % 2 == 0), near).argmax(-1)
    code = code + np.where(np.signbit(z), 8, 0)
    return code.reshape(np.shape(x)), np.where(finite, s + 127, 255)


def decode(code, scale):
    v = GRID[code & 7] * np.where(code >= 8, -1.0, 1.0)
    v = v.reshape(v.shape[:-1] + (-1, 32))
    f = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return (v * f[..., None]).reshape(code.shape)


def round4(x):
    """What rows x read back as."""
    return decode(*encode(x))


def places(d):
    """Byte offsets in a (page, kv head) block: K codes [slot][entry], V codes, K scales
    [slot][block], V scales."""
    t, c, b = np.arange(PAGE)[:, None], np.arange(d)[None], np.arange(d // 32)[None]
    k = ((c // (d // 4)) * PAGE + t) * (d // 8) + c % (d // 4) // 2
    v = 8 * d + (((t // 4) * 16 + c // (d // 16)) * 4 + t % 4) * (d // 32) + c % (d // 16) // 2
    return k, v, 16 * d + b * PAGE + t, 16 * d + d // 2 + ((t // 4) * (d // 32) + b) * 4 + t % 4


def read_pool(pool, d):
    """Pool bytes [pages][Hkv][17 d] -> K, V [pages][Hkv][16][d]."""
    k, v, ks, vs = places(d)
    odd = np.arange(d) % 2 == 1
    out = []
    for at, sc in ((k, ks), (v, vs)):
        byte = pool[:, :, at]
        out.append(decode(np.where(odd, byte >> 4, byte & 15).astype(np.int64), pool[:, :, sc].astype(np.int64)))
    return out


def write_slots(pool, page, slot, rows_k, rows_v):
    """Stores rows [n][Hkv][d] in slots (page[i], slot[i]) of the pool bytes, in place."""
    d = rows_k.shape[-1]
    places_ = places(d)
    for rows, at, sc in ((rows_k, places_[0], places_[2]), (rows_v, places_[1], places_[3])):
        code, scale = encode(rows)
        for i in range(len(page)):
            by = (code[i, :, 0::2] | (code[i, :, 1::2] << 4)).astype(np.uint8)
            pool[page[i]][:, at[slot[i], 0::2]] = by
            pool[page[i]][:, sc[slot[i]]] = scale[i].astype(np.uint8)


def gather(pool, table_row, n):
    """[pages][Hkv][16][...] -> the first n positions, [n][Hkv][...]."""
    pos = np.arange(n)
    return pool[table_row[pos // PAGE], :, pos % PAGE]


def attention(q, k, v, prefix, scale):
    """q [E][Hq][d], k, v [n][Hkv][d] -> out, lse, sum of weight |v|, largest sum |q k| scale."""
    e, hq, d = q.shape
    n, hkv, _ = k.shape
    g = hq // hkv
    qh = q.reshape(e, hkv, g, d)
    s = np.einsum("ehgd,nhd->ehgn", qh, k) * scale
    size = np.einsum("ehgd,nhd->ehgn", np.abs(qh), np.abs(k)).max() * scale if n else 0.0
    seen = np.arange(n)[None] <= prefix + np.arange(e)[:, None]
    s = np.where(seen[:, None, None], s, -np.inf)
    m = s.max(-1, keepdims=True)
    p = np.exp(s - m)
    l = p.sum(-1, keepdims=True)
    p = p / l
    out = np.einsum("ehgn,nhd->ehgd", p, v).reshape(e, hq, d)
    spread = np.einsum("ehgn,nhd->ehgd", p, np.abs(v)).reshape(e, hq, d)
    return out, (m + np.log(l))[..., 0].reshape(e, hq), spread, size


def out_bound(ref, spread):
    """Weights are rounded to bf16 (2^-8 of each, in the sum and in its divisor) and the result is;
    fp32 sums add far less."""
    return 2.0 ** -8 * np.abs(ref) * (1 + 2.0 ** -7) + 2 * 2.0 ** -8 * (1 + 2.0 ** -6) * spread + 1e-30


def score_bound(d, size):
    """fp32 sums of d exact products, the scaling to base 2 and back, and the exponential's argument."""
    return (d + 8) * 2.0 ** -24 * size + 2.0 ** -20


def mass(q, lse, k, prefix, scale):
    """Weights added to each key, [n][Hkv]."""
    e, hq, d = q.shape
    n, hkv, _ = k.shape
    s = np.einsum("ehgd,nhd->ehgn", q.reshape(e, hkv, -1, d), k) * scale - lse.reshape(e, hkv, -1)[..., None]
    seen = np.arange(n)[None] <= prefix + np.arange(e)[:, None]
    return np.where(seen[:, None, None], np.exp(s), 0.0).sum((0, 2)).T


def kept(sums, keep, recent):
    """Positions that one kv head keeps of `sums` [n]."""
    n = len(sums)
    w = np.where(np.isnan(sums[: n - recent]), -np.inf, sums[: n - recent])
    low = np.isnan(sums[: n - recent])  # below -inf
    order = np.lexsort((np.arange(n - recent), low, -w))
    return np.sort(np.concatenate((order[: keep - recent], np.arange(n - recent, n)))).astype(np.int64)
