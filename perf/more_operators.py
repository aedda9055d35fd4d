"""The operators of a step whose lengths live on the device and whose attention reads a budget of
blocks, as a rollout engine calls them.

A row is one query token: (row_task, row_pos, row_slot) on the device say whose it is, where in the
task's context it sits, and in which pool slot (page * 16 + slot) its K/V go.  A block is a page's 16
positions.

  map      from every task's cached and wanted lengths: pages taken from the free list or given
           back, the block table's new entries, and the rows of the tokens that come in
  append   the rows' K/V into their slots, and the key bounds of the pages that changed
  bounds   the key bounds of whole contexts: per page and kv head the least s in [-120, 122] with
           max|k| <= 127 * 2^s, hi = ceil(max over the page's positions of k / 2^s) and
           lo = floor(min of k / 2^s), entry by entry; s = 127, hi = lo = 0 where a key is not finite
  select   per row and kv head, the blocks to attend to: the first `sink`, the last `recent`, and
           the others with the highest score, `budget` in all, ascending, -1 behind them.  With
           t the least in [-120, 122] such that max|q| <= 127 * 2^t and c = q / 2^t to the nearest
           whole number (ties to even), the score of a block is the largest over the kv head's query
           heads of 2^clamp(s + t, -100, 100) * sum over entries of max(c * hi, c * lo): whole
           numbers times a power of two, so every score is exact and the choice has one answer
  attend   softmax attention of each row over the positions at or before its own in its blocks

`run` is the plain form unless `own` is set, with which it calls the framework.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
# (query heads, kv heads, head dim) of perf/cases.py
HEADS = ((28, 4, 128), (32, 8, 128), (64, 8, 128), (8, 2, 64), (8, 8, 128), (32, 2, 64))
MOST_BYTES = 2.1e9   # a drawn case does no more than the largest listed ones
MOST_FLOPS = 1.18e11
MOST_CONTEXT = 98304 + 2048
MOST_POOL = 9.0e9


def _case(name, kind, heads, tasks, ctx, new=(1, 1), budget=0, sink=0, recent=0, gone=0.0, free=1.1, lse=False,
          lens=1):
    """ctx: lo, hi of the cached context (select and attend: before the new tokens; bounds: all of it),
    uniform.  new: lo, hi of the new tokens, spread over their logarithm.  budget, sink, recent: blocks.
    gone: map, the share of tasks that end and give their pages back; free: the free pages as a share of
    those that the round takes."""
    c = {"kind": kind, "hq": heads[0], "hkv": heads[1], "d": heads[2], "tasks": tasks, "ctx_lo": ctx[0],
         "ctx_hi": ctx[1], "new_lo": new[0], "new_hi": new[1], "budget": budget, "sink": sink,
         "recent": recent, "gone": gone, "free": free, "lse": lse, "lens": lens}
    return dict(c, name=name) if name else c


def listed():
    return [
        # a decode round: one token a task, a page for every sixteenth
        _case("map_tokens", "map", HEADS[0], 175, (500, 3000)),
        # a scheduler round of the whole step's trajectories: observations arrive, some tasks end
        _case("map_round", "map", HEADS[0], 1056, (400, 3400), (1, 450), gone=0.1),
        # a decode round's tokens, each in the middle of a page
        _case("append_tokens", "append", HEADS[1], 256, (1024, 16384)),
        # a scheduler round's observations
        _case("append_observations", "append", HEADS[0], 64, (2048, 16384), (64, 2048)),
        # a few short contexts that were appended without bounds
        _case("bounds_few", "bounds", HEADS[3], 4, (300, 4000)),
        # a batch of paused tasks, after an eviction or a re-prefill
        _case("bounds_paused", "bounds", HEADS[0], 64, (2048, 16384)),
        # the tail of a rollout step: a few trajectories still generate
        _case("select_few", "select", HEADS[0], 4, (2048, 16384), budget=64, sink=1, recent=2),
        # a full decode batch
        _case("select_batch", "select", HEADS[1], 256, (1024, 32768), budget=128, sink=1, recent=4),
        # long-horizon agents: an observation over a very long context, each token with blocks of its own
        _case("select_chunk", "select", HEADS[2], 8, (32768, 98304), (64, 512), budget=128, sink=1, recent=4),
        # as select_few
        _case("attend_few", "attend", HEADS[0], 4, (2048, 16384), budget=64, sink=1, recent=2, lse=True),
        # as select_batch
        _case("attend_batch", "attend", HEADS[1], 256, (1024, 16384), budget=128, sink=1, recent=4),
        # as select_chunk
        _case("attend_chunk", "attend", HEADS[2], 8, (32768, 98304), (64, 512), budget=128, sink=1, recent=4),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    """One more case: a kind, a model shape, a batch, lengths and a budget over the listed ranges."""
    while True:
        kind = rng.choice(("map", "append", "bounds", "select", "select", "attend", "attend"))
        heads = rng.choice(HEADS[:3] + HEADS)
        lo = _log_int(rng, 20, 65536)
        ctx = (lo, int(lo * rng.uniform(1.0, 8.0)))
        n = _log_int(rng, 1, {"map": 450, "append": 2048, "bounds": 1}.get(kind, 512))
        if kind in ("select", "attend") and rng.random() < 0.5:
            n = 1
        new = (n, int(n * rng.uniform(1.0, 4.0)) if n > 1 else n)
        budget = _log_int(rng, 4, 512) if kind in ("select", "attend") else 0
        c = _case("", kind, heads, _log_int(rng, 1, 1056 if kind == "map" else 256), ctx, new, budget,
                  sink=rng.randint(0, 2) if budget else 0, recent=rng.randint(0, min(8, budget - 2)) if budget else 0,
                  gone=round(rng.uniform(0.0, 0.5), 2) if kind == "map" else 0.0,
                  free=round(rng.uniform(0.5, 1.5), 2) if kind == "map" else 1.1,
                  lse=kind == "attend" and rng.random() < 0.5, lens=rng.randrange(1 << 30))
        ln = _lengths(c)
        w = work(c)
        if kind == "select" and _pages(ln["total"]).max() < 2 * budget:  # nothing to choose
            continue
        if w["bytes"] <= MOST_BYTES and w["flops"] <= MOST_FLOPS and ln["total"].max() <= MOST_CONTEXT \
                and ln["new"].sum() <= (1 << 16 if kind in ("map", "append") else 2048) and _pool_bytes(c, ln) <= MOST_POOL:
            return c


def _lengths(case):
    """Host lengths of every task: cached, new tokens, their sum; map: what is wanted."""
    rng = np.random.default_rng([2608, 10402, 5, case["lens"]])
    n = case["tasks"]
    prefix = rng.integers(case["ctx_lo"], case["ctx_hi"], n, endpoint=True).astype(np.int32)
    if case["kind"] == "bounds":
        new = np.zeros(n, np.int32)
    else:
        new = np.exp(rng.uniform(math.log(case["new_lo"]), math.log(case["new_hi"] + 1), n))
        new = np.clip(new.astype(np.int32), case["new_lo"], case["new_hi"])
    gone = rng.random(n) < case["gone"]
    new = np.where(gone, 0, new).astype(np.int32)
    total = (prefix + new).astype(np.int32)
    return {"prefix": prefix, "new": new, "total": total, "want": np.where(gone, 0, total).astype(np.int32)}


def _pages(n):
    return -(-np.asarray(n, np.int64) // PAGE)


def _pool_bytes(case, ln):
    pages, hkv, d = float(_pages(ln["total"]).sum()), case["hkv"], case["d"]
    return pages * hkv * {"map": 0.0, "append": 0.0, "bounds": 32.0 * d, "select": 2.0 * d, "attend": 64.0 * d}[case["kind"]]


def _attended(case, ln):
    """Per task: visible blocks of the last row, and positions that all rows attend to (at most)."""
    blocks = _pages(ln["total"]).astype(np.float64)
    keys = np.minimum(ln["total"].astype(np.float64), PAGE * float(case["budget"]))
    return blocks, ln["new"] * keys


def work(case):
    """Each input read once and each output written once.  select: 4 d operations a query head and block;
    attend: 4 d flops a query head and attended position, and at least one row's blocks of every task."""
    ln = _lengths(case)
    hq, hkv, d, kind = case["hq"], case["hkv"], case["d"], case["kind"]
    rows, n = float(ln["new"].sum()), case["tasks"]
    have, want = _pages(ln["prefix"]), _pages(ln["want"])
    if kind == "map":  # lengths read and written; a page moves: one id read, one written; a row: 16 bytes
        return {"bytes": 16.0 * n + 8.0 * float(np.abs(want - have).sum()) + 16.0 * rows, "flops": 0.0}
    if kind == "append":  # rows read and written, the other keys of the first page read, bounds written
        older = float((ln["prefix"] % PAGE).sum())
        changed = float((_pages(ln["total"]) - ln["prefix"] // PAGE).sum())
        return {"bytes": rows * hkv * 8.0 * d + rows * 8.0 + older * hkv * 2.0 * d + changed * hkv * (2.0 * d + 1.0),
                "flops": 0.0}
    if kind == "bounds":
        pages = float(_pages(ln["total"]).sum())
        return {"bytes": float(ln["total"].sum()) * hkv * 2.0 * d + pages * (hkv * (2.0 * d + 1.0) + 4.0), "flops": 0.0}
    blocks, keys = _attended(case, ln)
    if kind == "select":
        p, e = ln["prefix"].astype(np.float64), ln["new"].astype(np.float64)
        pairs = float((e * (p + (e + 1) / 2) / PAGE).sum())
        nbytes = float(blocks.sum()) * (hkv * (2.0 * d + 1.0) + 4.0) + rows * (hq * 2.0 * d + 8.0 + hkv * case["budget"] * 4.0)
        return {"bytes": nbytes, "flops": 4.0 * d * hq * pairs}
    once = float(np.minimum(ln["total"], PAGE * case["budget"]).sum())
    nbytes = once * hkv * 4.0 * d + rows * (hq * 4.0 * d + 8.0 + hkv * case["budget"] * 4.0 + (hq * 4.0 if case["lse"] else 0.0))
    return {"bytes": nbytes, "flops": 4.0 * d * hq * float(keys.sum())}


# ---- inputs ----------------------------------------------------------------------------------

class _State:
    pass


def _rows_of(ln):
    """Task and position of every new token, in task order (host)."""
    task = np.repeat(np.arange(ln["new"].size), ln["new"])
    start = np.repeat(ln["prefix"] - (np.cumsum(ln["new"]) - ln["new"]), ln["new"])
    return task.astype(np.int32), (start + np.arange(task.size)).astype(np.int32)


def _key_bounds(k):
    """hi, lo and s of pages k [..., 16, d] (fp32) of which every position counts."""
    hi, lo = k.amax(-2), k.amin(-2)
    top = torch.maximum(hi.abs(), lo.abs()).amax(-1)
    ok = torch.isfinite(k).all(-1).all(-1)
    s = _unit(torch.where(ok, top, 1.0))
    two = torch.ldexp(torch.ones_like(hi, dtype=torch.float64), -s[..., None].double())
    whole = ok[..., None]
    hi = torch.where(whole, torch.ceil(hi.double() * two), 0.0).to(torch.int8)
    lo = torch.where(whole, torch.floor(lo.double() * two), 0.0).to(torch.int8)
    return hi, lo, torch.where(ok, s, 127).to(torch.int8)


def _unit(top):
    """The least s in [-120, 122] with top <= 127 * 2^s."""
    mant, ex = torch.frexp(top)  # top = mant 2^ex, mant in [1/2, 1)
    s = ex - 7 + (mant > 127.0 / 128.0)
    return torch.where(top > 0, s, -120).clamp(-120, 122)


def _choose(score, blocks, budget, sink, recent):
    """Of `blocks` [rows] leading entries of score [rows, heads, n]: the first sink, the last recent and
    the highest of the others (equal scores: the earlier), ascending, -1 behind them."""
    n = score.shape[-1]
    at = torch.arange(n, device=score.device)
    last = blocks[:, None, None]
    always = (at < sink) | (at >= last - recent)
    key = torch.where(always, math.inf, score)
    key = torch.where(at < last, key, -math.inf)
    # (two stable sorts keep what is always taken before a score of +inf, and both before what is not there)
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices
    rank = (always & (at < last)).to(torch.int8) - (at >= last).to(torch.int8)
    order = order.gather(-1, torch.sort(rank.expand(score.shape).gather(-1, order), dim=-1, descending=True, stable=True).indices)
    order = order[..., :budget]
    got = torch.where(order < last, order, n)
    got = torch.sort(got, dim=-1).values
    got = torch.where(got < n, got, -1)
    return torch.nn.functional.pad(got, (0, budget - got.shape[-1]), value=-1).to(torch.int32)


def prepare(case, seed):
    """Pools whose pages hold the contexts (scattered over 1.1 times the pages in use), block tables,
    key bounds, the rows and what else the kind takes."""
    dev = torch.device("cuda")
    ln = _lengths(case)
    hq, hkv, d, n, kind = case["hq"], case["hkv"], case["d"], case["tasks"], case["kind"]
    rng = np.random.default_rng([int(seed), 5, case["lens"]])
    gen = torch.Generator(device=dev)
    gen.manual_seed((int(seed) * 1000003 + 17) % (1 << 62))

    def up(x):
        return torch.from_numpy(np.ascontiguousarray(x)).to(dev)

    def normal(*shape):
        return torch.empty(shape, dtype=torch.bfloat16, device=dev).normal_(generator=gen)

    s = _State()
    s.case, s.ln, s.kv = case, ln, None
    task, pos = _rows_of(ln)
    s.rows = int(task.size)
    # first logical page that the kind touches (append leaves the others alone)
    first = ln["prefix"].astype(np.int64) // PAGE if kind == "append" else np.zeros(n, np.int64)
    held = _pages(ln["prefix"]) if kind == "map" else _pages(ln["total"])
    used = int((held - first).sum())
    taken = int(np.maximum(0, _pages(ln["want"]) - _pages(ln["prefix"])).sum())
    pool = int(used * 1.1) + 1
    if kind == "map":
        pool = used + int(taken * case["free"]) + 1
    order = rng.permutation(pool).astype(np.int32)
    table, at = np.zeros((n, int(_pages(ln["total"]).max())), np.int32), 0
    for b in range(n):
        m = int(held[b] - first[b])
        table[b, first[b]: held[b]] = order[at: at + m]
        at += m
    s.host_table, s.table, s.pool_pages = table, up(table), pool
    s.row_task, s.row_pos = up(task), up(pos)
    if kind == "map":
        s.lens, s.want = up(ln["prefix"]), up(ln["want"])
        free = order[at:]
        s.free_pages = torch.full((pool,), -1, dtype=torch.int32, device=dev)
        s.free_pages[: free.size] = up(free)
        s.free_count = up(np.array([free.size], np.int32))
        s.lens_out, s.free_count_out = torch.empty_like(s.lens), torch.empty_like(s.free_count)
        s.row_start = torch.empty(n + 1, dtype=torch.int32, device=dev)
        s.row_slot = torch.empty(s.rows, dtype=torch.int64, device=dev)
        return s
    if kind == "append":
        s.row_slot = up(table[task, pos // PAGE].astype(np.int64) * PAGE + pos % PAGE)
        s.k_pool, s.v_pool = normal(pool, hkv, PAGE, d), normal(pool, hkv, PAGE, d)
        s.k, s.v = normal(s.rows, hkv, d), normal(s.rows, hkv, d)
    if kind == "bounds":
        s.lens = up(ln["total"])
        s.k_pool = normal(pool, hkv, PAGE, d)
    if kind in ("append", "bounds"):
        s.bounds = torch.zeros((pool, hkv, 2, d), dtype=torch.int8, device=dev)
        s.units = torch.zeros((pool, hkv), dtype=torch.int8, device=dev)
        return s
    s.q = normal(s.rows, hq, d)
    if kind == "select":
        # every page one of 8192, whose keys share a direction of their own; equal pages tie
        bank = normal(8192, PAGE, d).float() + normal(8192, 1, d).float()
        hi, lo, unit = _key_bounds(bank)
        bank = torch.stack((hi, lo), 1)
        pick = torch.randint(0, 8192, (pool, hkv), generator=gen, device=dev)
        s.bounds, s.units = bank[pick], unit[pick]
        return s
    s.k_pool, s.v_pool = normal(pool, hkv, PAGE, d), normal(pool, hkv, PAGE, d)
    s.sel = torch.empty((s.rows, hkv, case["budget"]), dtype=torch.int32, device=dev)
    r0 = 0
    for b in range(n):  # blocks of a task that its rows like in common, and each a little by itself
        e, m = int(ln["new"][b]), int(_pages(ln["total"][b]))
        like = torch.empty((1, hkv, m), device=dev).normal_(generator=gen)
        step = max(1, (1 << 26) // (hkv * m))
        for r in range(0, e, step):
            k = min(step, e - r)
            like_r = like + 0.3 * torch.empty((k, hkv, m), device=dev).normal_(generator=gen)
            blocks = s.row_pos[r0 + r: r0 + r + k].long() // PAGE + 1
            s.sel[r0 + r: r0 + r + k] = _choose(like_r, blocks, case["budget"], case["sink"], case["recent"])
        r0 += e
    s.lse = torch.empty((s.rows, hq), dtype=torch.float32, device=dev) if case["lse"] else None
    return s


# ---- the plain form ---------------------------------------------------------------------------

def _excl(x):
    return torch.cumsum(x, 0) - x


def _plain_map(s):
    ln, dev = s.ln, s.table.device
    lens, want = s.lens.long(), s.want.long()
    have, need = (lens + PAGE - 1) // PAGE, (want + PAGE - 1) // PAGE
    # pages of the tasks that shrink go onto the stack, in task order
    give = (have - need).clamp(min=0)
    n_give = int(np.maximum(0, _pages(ln["prefix"]) - _pages(ln["want"])).sum())
    who = torch.repeat_interleave(torch.arange(lens.numel(), device=dev), give, output_size=n_give)
    which = need[who] + torch.arange(n_give, device=dev) - _excl(give)[who]
    count = s.free_count[0].long()
    s.free_pages[count + torch.arange(n_give, device=dev)] = s.table[who, which]
    have_free = count + n_give
    # tasks that grow take theirs from its top, while there are enough
    grow = (want - lens).clamp(min=0)
    take = torch.where(grow > 0, need - have, 0)
    ok = (take == 0) | (torch.cumsum(take, 0) <= have_free)
    take = torch.where(ok, take, 0)
    n_take = int(np.maximum(0, _pages(ln["want"]) - _pages(ln["prefix"])).sum())
    j = torch.arange(n_take, device=dev)
    there = j < take.sum()
    who = torch.searchsorted(torch.cumsum(take, 0), j, right=True).clamp(max=lens.numel() - 1)
    which = have[who] + j - _excl(take)[who]
    page = s.free_pages[(have_free - 1 - j).clamp(min=0)]
    who, which = torch.where(there, who, 0), torch.where(there, which, 0)
    s.table[who, which] = torch.where(there, page, s.table[0, 0])
    s.lens_out.copy_(torch.where(ok, want, lens))
    s.free_count_out.copy_((have_free - take.sum())[None])
    s.row_start[0] = 0
    s.row_start[1:] = torch.cumsum(grow, 0)
    who = torch.repeat_interleave(torch.arange(lens.numel(), device=dev), grow, output_size=s.rows)
    pos = lens[who] + torch.arange(s.rows, device=dev) - s.row_start[who]
    slot = s.table[who, pos // PAGE].long() * PAGE + pos % PAGE
    s.row_task.copy_(torch.where(ok[who], who, -1))
    s.row_pos.copy_(torch.where(ok[who], pos, -1))
    s.row_slot.copy_(torch.where(ok[who], slot, -1))


def _map_outputs(s):
    return {"lens": s.lens_out, "table": s.table, "free_pages": s.free_pages, "free_count": s.free_count_out,
            "row_start": s.row_start, "row_task": s.row_task, "row_pos": s.row_pos, "row_slot": s.row_slot}


def _bounds_of_pages(s, page, count):
    """Bounds of the first count [m] slots of pages page [m], into the state's."""
    for i in range(0, page.numel(), 4096):
        p, c = page[i:i + 4096], count[i:i + 4096]
        slot = torch.minimum(torch.arange(PAGE, device=p.device), c[:, None] - 1)  # past count: the last again
        k = s.k_pool[p].float().gather(2, slot[:, None, :, None].expand(-1, s.case["hkv"], -1, s.case["d"]))
        hi, lo, unit = _key_bounds(k)
        s.bounds[p, :, 0], s.bounds[p, :, 1], s.units[p] = hi, lo, unit


def _plain_append(s):
    page, slot = s.row_slot // PAGE, s.row_slot % PAGE
    s.k_pool[page, :, slot] = s.k
    s.v_pool[page, :, slot] = s.v
    # the last row of each page, up to which it is filled
    last = torch.ones_like(page, dtype=torch.bool)
    last[:-1] = page[1:] != page[:-1]
    count = torch.zeros(s.pool_pages, dtype=torch.int64, device=page.device)
    count.scatter_reduce_(0, torch.where(last, page, s.pool_pages - 1), torch.where(last, slot + 1, 0), "amax")
    changed = torch.nonzero(count)[:, 0]
    _bounds_of_pages(s, changed, count[changed])
    return {"k_pool": s.k_pool, "v_pool": s.v_pool, "bounds": s.bounds, "units": s.units}


def _plain_bounds(s):
    task = torch.from_numpy(np.repeat(np.arange(s.case["tasks"]), _pages(s.ln["total"]))).to(s.table.device)
    m = (s.lens.long() + PAGE - 1) // PAGE
    lp = torch.arange(task.numel(), device=task.device) - _excl(m)[task]
    _bounds_of_pages(s, s.table[task, lp].long(), (s.lens[task] - PAGE * lp).clamp(max=PAGE))
    return {"bounds": s.bounds, "units": s.units}


def _plain_select(s):
    c, ln = s.case, s.ln
    hq, hkv, d, g = c["hq"], c["hkv"], c["d"], c["hq"] // c["hkv"]
    sel = torch.empty((s.rows, hkv, c["budget"]), dtype=torch.int32, device=s.q.device)
    r0 = 0
    for b in range(c["tasks"]):
        e, m = int(ln["new"][b]), int(_pages(ln["total"][b]))
        page = s.table[b, :m].long()
        w = s.bounds[page].float().flatten(2).permute(1, 2, 0).contiguous()  # [hkv, hi and lo, blocks]
        unit = s.units[page].t()[:, None, :]
        step = max(1, (1 << 26) // (hq * m))
        for r in range(r0, r0 + e, step):
            k = min(step, r0 + e - r)
            q = s.q[r: r + k].float().view(k, hkv, g, d).transpose(0, 1).reshape(hkv, k * g, d)
            t = _unit(q.abs().amax(-1))
            code = torch.round(torch.ldexp(q, -t[..., None]))
            both = torch.cat((code.clamp(min=0.0), code.clamp(max=0.0)), -1)
            # (whole numbers below 2^24: exact in any order)
            x = torch.bmm(both, w)
            x = torch.ldexp(x, (unit + t[..., None]).clamp(-100, 100))
            x = torch.where(unit == 127, math.inf, x)
            x = x.view(hkv, k, g, m).amax(2).transpose(0, 1)
            blocks = s.row_pos[r: r + k].long() // PAGE + 1
            sel[r: r + k] = _choose(x, blocks, c["budget"], c["sink"], c["recent"])
        r0 += e
    return {"sel": sel}


def _plain_attend(s):
    c = s.case
    hq, hkv, d, g, k = c["hq"], c["hkv"], c["d"], c["hq"] // c["hkv"], c["budget"]
    dev = s.q.device
    out = torch.empty((s.rows, hq, d), dtype=torch.bfloat16, device=dev)
    lse = torch.empty((s.rows, hq), dtype=torch.float32, device=dev)
    heads = torch.arange(hkv, device=dev)[None, :, None]
    step = max(1, (1 << 27) // (hkv * k * PAGE * d))
    for r in range(0, s.rows, step):
        m = min(step, s.rows - r)
        sel = s.sel[r: r + m].long()
        page = s.table[s.row_task[r: r + m].long()[:, None, None], sel.clamp(min=0)].long()
        key = s.k_pool[page, heads].flatten(2, 3).float().view(m * hkv, k * PAGE, d)
        val = s.v_pool[page, heads].flatten(2, 3).float().view(m * hkv, k * PAGE, d)
        at = (sel[..., None] * PAGE + torch.arange(PAGE, device=dev)).flatten(2)
        seen = (sel >= 0).repeat_interleave(PAGE, 2) & (at <= s.row_pos[r: r + m].long()[:, None, None])
        q = s.q[r: r + m].float().view(m * hkv, g, d).transpose(1, 2).contiguous()
        x = torch.bmm(key, q).transpose(1, 2).contiguous() * (1.0 / math.sqrt(d))
        x.masked_fill_(~seen.view(m * hkv, 1, k * PAGE), -math.inf)
        mx = x.amax(-1, keepdim=True)
        x = (x - mx).exp_()
        l = x.sum(-1, keepdim=True)
        lse[r: r + m] = (mx + l.log()).view(m, hq)
        out[r: r + m] = (torch.bmm(x, val) / l).view(m, hq, d).to(torch.bfloat16)
    return {"out": out, "lse": lse} if c["lse"] else {"out": out}


# ---- one pass ---------------------------------------------------------------------------------

def _handle(s):
    import paper_2608_10402_amd as tide

    c = s.case
    kv = tide.PagedKV(1, c["hq"], c["hkv"], c["d"], s.host_table, fill_canary=False)
    if hasattr(s, "k_pool"):
        kv.k_pool, kv.v_pool = s.k_pool, getattr(s, "v_pool", s.k_pool)
    return kv


def run(s):
    c, kind = s.case, s.case["kind"]
    if not own:
        if kind == "map":
            _plain_map(s)
            return _map_outputs(s)
        return {"append": _plain_append, "bounds": _plain_bounds, "select": _plain_select,
                "attend": _plain_attend}[kind](s)
    if s.kv is None:
        s.kv = _handle(s)
    kv = s.kv
    if kind == "map":
        import paper_2608_10402_amd as tide

        tide.tide_page_map(s.lens, s.want, s.table, s.free_pages, s.free_count, s.lens_out, s.free_count_out,
                           s.row_start, s.row_task, s.row_pos, s.row_slot, kv.dims)
        return _map_outputs(s)
    if kind == "append":
        kv.append_slots(s.k, s.v, s.row_slot, (s.bounds, s.units))
        return {"k_pool": s.k_pool, "v_pool": s.v_pool, "bounds": s.bounds, "units": s.units}
    if kind == "bounds":
        kv.key_bounds(s.lens, (s.bounds, s.units))
        return {"bounds": s.bounds, "units": s.units}
    if kind == "select":
        return {"sel": kv.select_blocks(s.q, s.row_task, s.row_pos, (s.bounds, s.units), c["budget"], c["sink"],
                                        c["recent"])}
    out = kv.sparse(s.q, s.row_task, s.row_pos, s.sel, lse=s.lse)
    return {"out": out, "lse": s.lse} if c["lse"] else {"out": out}


# ---- the definition in 64 bits --------------------------------------------------------------------

def _exact_map(s):
    """One task after the other, as a host's allocator would."""
    ln = s.ln
    table, free = s.host_table.copy(), s.free_pages.cpu().numpy()
    top = int(s.free_count[0])
    lens, want = ln["prefix"].astype(np.int64), ln["want"].astype(np.int64)
    out, row_start = lens.copy(), np.zeros(lens.size + 1, np.int64)
    for b in range(lens.size):
        if want[b] < lens[b]:
            for i in range(int(_pages(want[b])), int(_pages(lens[b]))):
                free[top] = table[b, i]
                top += 1
            out[b] = want[b]
    rows, short = [], False
    for b in range(lens.size):
        row_start[b + 1] = row_start[b] + max(0, want[b] - lens[b])
        if want[b] <= lens[b]:
            continue
        first, end = int(_pages(lens[b])), int(_pages(want[b]))
        if end > first and (short or end - first > top):
            short = True
            rows += [(-1, -1, -1)] * int(want[b] - lens[b])
            continue
        for i in range(first, end):
            top -= 1
            table[b, i] = free[top]
        out[b] = want[b]
        rows += [(b, p, int(table[b, p // PAGE]) * PAGE + p % PAGE) for p in range(int(lens[b]), int(want[b]))]
    rows = np.array(rows, np.int64).reshape(-1, 3)
    got = {"lens": out, "table": table, "free_pages": free, "free_count": np.array([top]), "row_start": row_start,
           "row_task": rows[:, 0], "row_pos": rows[:, 1], "row_slot": rows[:, 2]}
    like = _map_outputs(s)
    return {k: torch.from_numpy(np.ascontiguousarray(v)).to(like[k].dtype) for k, v in got.items()}


def _exact_unit(top):
    """The least s in [-120, 122] with top <= 127 * 2^s, by trying them."""
    s = torch.full(top.shape, 122, dtype=torch.int64, device=top.device)
    for e in range(121, -121, -1):
        s = torch.where(top <= 127.0 * 2.0 ** e, e, s)
    return s


def _exact_bounds(s, filled):
    """Bounds of the pages with filled[page] > 0 slots, from 64-bit keys, slot by slot."""
    bounds, units = s.bounds.clone(), s.units.clone()
    pages = torch.nonzero(filled)[:, 0]
    for i in range(0, pages.numel(), 8192):
        p = pages[i:i + 8192]
        hi = lo = s.k_pool[p, :, 0].double()
        for t in range(1, PAGE):
            k = s.k_pool[p, :, t].double()
            there = (filled[p] > t)[:, None, None]
            hi = torch.where(there & (k > hi), k, hi)
            lo = torch.where(there & (k < lo), k, lo)
        unit = _exact_unit(torch.maximum(hi.abs(), lo.abs()).amax(-1))
        two = torch.exp2(unit.double())[..., None]
        bounds[p, :, 0] = torch.ceil(hi / two).to(torch.int8)
        bounds[p, :, 1] = torch.floor(lo / two).to(torch.int8)
        units[p] = unit.to(torch.int8)
    return bounds, units


def exact(case, seed):
    s = prepare(case, seed)
    ln, kind, hq, hkv, d = s.ln, case["kind"], case["hq"], case["hkv"], case["d"]
    g, dev = hq // hkv, s.table.device
    if kind == "map":
        return _exact_map(s)
    if kind in ("append", "bounds"):
        filled = np.zeros(s.pool_pages, np.int64)
        for b in range(case["tasks"]):
            n = int(ln["total"][b])
            for i in range(int(ln["prefix"][b]) // PAGE if kind == "append" else 0, int(_pages(n))):
                filled[s.host_table[b, i]] = min(PAGE, n - PAGE * i)
        if kind == "append":
            task, pos = _rows_of(ln)
            for h in range(hkv):
                for pool, new in ((s.k_pool, s.k), (s.v_pool, s.v)):
                    flat = pool[:, h].reshape(-1, d)
                    flat[torch.from_numpy(s.host_table[task, pos // PAGE].astype(np.int64) * PAGE + pos % PAGE).to(dev)] = new[:, h]
                    pool[:, h] = flat.view(-1, PAGE, d)
        bounds, units = _exact_bounds(s, torch.from_numpy(filled).to(dev))
        got = {"bounds": bounds, "units": units}
        return dict(got, k_pool=s.k_pool, v_pool=s.v_pool) if kind == "append" else got
    budget, sink, recent = case["budget"], case["sink"], case["recent"]
    if kind == "select":
        sel = torch.full((s.rows, hkv, budget), -1, dtype=torch.int32)
        r0 = 0
        for b in range(case["tasks"]):
            e, m = int(ln["new"][b]), int(_pages(ln["total"][b]))
            page = s.table[b, :m].long()
            for h in range(hkv):
                hi, lo = s.bounds[page, h, 0].double(), s.bounds[page, h, 1].double()
                unit = s.units[page, h].double()
                for r in range(r0, r0 + e, 256):
                    k = min(256, r0 + e - r)
                    q = s.q[r: r + k, h * g:(h + 1) * g].double().reshape(k * g, d)
                    t = _exact_unit(q.abs().amax(-1)).double()
                    code = q / torch.exp2(t)[:, None]
                    low = torch.floor(code)
                    up = (code - low > 0.5) | ((code - low == 0.5) & (torch.remainder(low, 2.0) == 1.0))
                    code = low + up
                    # max(c hi, c lo) = c (hi + lo) / 2 + |c| (hi - lo) / 2
                    x = code.mm((0.5 * (hi + lo)).t().contiguous()) + code.abs().mm((0.5 * (hi - lo)).t().contiguous())
                    x = x * torch.exp2((unit[None] + t[:, None]).clamp(-100, 100))
                    x = x.view(k, g, m).amax(1).cpu().numpy()
                    for i in range(k):
                        nb = int(s.ln["prefix"][b] + r - r0 + i) // PAGE + 1
                        if nb <= budget:
                            pick = np.arange(nb)
                        else:
                            mid = x[i, sink: nb - recent]
                            best = sink + np.argsort(-mid, kind="stable")[: budget - sink - recent]
                            pick = np.sort(np.concatenate((np.arange(sink), best, np.arange(nb - recent, nb))))
                        sel[r + i, h, : pick.size] = torch.from_numpy(pick.astype(np.int32))
            r0 += e
        return {"sel": sel}
    out = torch.empty((s.rows, hq, d), dtype=torch.float64, device=dev)
    lse = torch.empty((s.rows, hq), dtype=torch.float64, device=dev)
    host_sel = s.sel.cpu().numpy()
    task, pos = _rows_of(ln)
    for r in range(s.rows):
        for h in range(hkv):
            blocks = host_sel[r, h]
            blocks = blocks[blocks >= 0].astype(np.int64)
            page = torch.from_numpy(s.host_table[task[r], blocks].astype(np.int64)).to(dev)
            n = min(PAGE * blocks.size, int(PAGE * (blocks.size - 1) + pos[r] - PAGE * blocks[-1] + 1))
            key = s.k_pool[page, h].reshape(-1, d)[:n].double()
            val = s.v_pool[page, h].reshape(-1, d)[:n].double()
            x = s.q[r, h * g:(h + 1) * g].double().mm(key.t().contiguous()) / math.sqrt(d)
            z = torch.logsumexp(x, -1)
            out[r, h * g:(h + 1) * g] = torch.exp(x - z[:, None]).mm(val)
            lse[r, h * g:(h + 1) * g] = z
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}
