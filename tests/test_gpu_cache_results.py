"""Results of the 4-bit cache, attention mass and eviction in calls that other tests only make, or do not
make: bad page ids, an extend of several rounds, evictions without a list of positions, groups that
share their prompt's pages (needs an MI355X)."""
import numpy as np
import pytest
import torch

import cache_reference as R
import paper_2608_10402_amd as tide
from test_gpu_evict import Cache
from test_gpu_kv4 import PAGE, Filled, check, host, rows_to_dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("call", ["decode", "decode_append", "extend_few", "extend"])
def test_slots_of_bad_pages_are_zeros_and_stay(call, d):
    """Attention reads zeros for them; a token that would be appended to one goes nowhere."""
    f = Filled(17, [100, 60], 16, 2, d)
    pool = f.kv.pool.clone()
    bad = f.table.copy()
    bad[0, 2], bad[1, 3] = -5, 1 << 30
    f.kv.set_block_table(bad)
    k, v = ([np.array(f.task(b)[i]) for b in range(2)] for i in range(2))
    new = [R.bf16(f.rng.standard_normal((2, 2, d))) for _ in range(2)]
    if call == "decode_append":
        k[0][99], v[0][99] = R.round4(new[0][0]), R.round4(new[1][0])
    for x in (k, v):
        x[0][32:48] = 0
        x[1][48:60] = 0  # the newest token's slot of task 1 among them
    extend = {"extend_few": [2, 2], "extend": [90, 50]}.get(call, [1, 1])
    prefix = f.lens - np.array(extend, np.int32)
    if call.startswith("extend"):
        info = tide.tide_plan_info_get(tide.TIDE_OP_KV4_EXTEND, prefix, extend, f.kv.dims)
        assert (info["run_steps"] == 0) == (call == "extend")
    q = f.queries(sum(extend))
    lse = torch.full((len(q), 16), float("nan"), device="cuda")
    if call == "decode":
        out = f.kv.decode(rows_to_dev(q), f.lens, lse=lse)
    elif call == "decode_append":
        out = f.kv.decode_append(rows_to_dev(q), rows_to_dev(new[0]), rows_to_dev(new[1]), f.lens, lse=lse)
    else:
        out = f.kv.extend(rows_to_dev(q), prefix, extend, lse=lse)
    at = 0
    for b, e in enumerate(extend):
        check(host(out)[at:at + e], host(lse)[at:at + e],
              R.attention(q[at:at + e], k[b], v[b], prefix[b], d ** -0.5))
        at += e
    want = pool.cpu().numpy()
    if call == "decode_append":
        R.write_slots(want, [bad[0, 6]], [99 % PAGE], new[0][:1], new[1][:1])
    assert np.array_equal(f.kv.pool.cpu().numpy(), want)


def test_extend_of_two_rounds():
    """More unpacked pages than a round holds (104 at 2,500 kv heads): the rows and log-sum-exps of both
    rounds, tasks without new tokens between them."""
    hkv, d = 2500, 64
    prefix, extend = np.array([400, 30, 300, 0, 410, 7], np.int32), np.array([240, 0, 250, 0, 235, 0], np.int32)
    rng, gen = np.random.default_rng(6), torch.Generator(device="cuda").manual_seed(6)
    total = prefix + extend
    pages = -(-total // PAGE)
    assert 64 < pages[0] + pages[2] <= 104 < pages[0] + pages[2] + pages[4]  # a page is 10.24 MB of bf16 K and V
    table = np.full((6, pages.max()), 1 << 20, np.int32)
    order, at = rng.permutation(int(pages.sum()) + 2), 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n]
        at += n
    kv = tide.PagedKV4(len(order), hkv, hkv, d, table, fill_canary=False)
    kv.pool.random_(0, 256, generator=gen)
    kv.pool[:, :, 16 * d:] = kv.pool[:, :, 16 * d:] % 4 + 125  # scales 2^-2 .. 2
    assert (1 << 29) < tide.tide_workspace_size(tide.TIDE_OP_KV4_EXTEND, prefix, extend, kv.dims) < (1 << 30) + (1 << 27)
    rows = int(extend.sum())
    q = torch.empty((rows, hkv, d), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    guard = torch.full((rows + 2, hkv, d), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((rows + 2, hkv), 7.0, device="cuda")
    kv.extend(q, prefix, extend, out=guard[1:-1], lse=lse[1:-1])
    assert (guard[[0, -1]] == 7).all() and (lse[[0, -1]] == 7).all()
    heads = [0, 7, 1300, hkv - 1]
    k, v = R.read_pool(kv.pool[:, heads].cpu().numpy(), d)
    q, out, z = host(q[:, heads]), host(guard[1:-1, heads]), host(lse[1:-1, heads])
    at = 0
    for b, e in enumerate(extend):
        if e:
            own = (R.gather(x, table[b], total[b]) for x in (k, v))
            check(out[at:at + e], z[at:at + e], R.attention(q[at:at + e], *own, prefix[b], d ** -0.5))
        at += e


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("inplace", [True, False])
def test_eviction_without_the_list_of_positions(bits, inplace):
    """kept = NULL: pools and sums are what they are with it."""
    got = []
    for listed in (True, False):
        c = Cache(29, [500, 90, 16], 8, 2, 128, bits, extra=40)
        free = np.array([p for p in range(c.sums.shape[0]) if p not in set(c.table.ravel())], np.int32)
        new = None if inplace else torch.from_numpy(free[:36].reshape(3, 12)).cuda()
        keep, recent, mass = [180, 90, 3], [16, 8, 0], c.mass()
        kept = torch.empty((273, 2), dtype=torch.int32, device="cuda") if listed else None
        ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
        args = (mass, c.kv.block_table, c.lens, keep, c.kv.dims, recent, new, kept, ws)
        if bits == 4:
            tide.tide_kv4_evict(c.kv.pool, *args)
        else:
            tide.tide_kv_evict(c.kv.k_pool, c.kv.v_pool, *args)
        got.append([mass] + ([c.kv.pool] if bits == 4 else [c.kv.k_pool, c.kv.v_pool]))
    for x, y in zip(*got):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@pytest.mark.parametrize("bits", [16, 4])
def test_sums_of_a_group_that_shares_its_prompt(bits):
    """Tasks that map the same pages, in calls of their own one after the other: the shared keys' sums are
    those of all their rows, each task's own keys' those of its own."""
    hq, hkv, d, prompt, own = 8, 2, 128, 96, [20, 33, 5]
    c = Cache(31, [prompt] + own, hq, hkv, d, bits)
    shared = c.table[0, : prompt // PAGE]
    table = np.stack([np.concatenate((shared, c.table[1 + b])) for b in range(3)]).astype(np.int32)
    mass, want, bound = c.mass(), c.sums.astype(np.float64), np.zeros(c.sums.shape)
    for b, n in enumerate(own):
        k, v = (np.concatenate((x, y)) for x, y in zip(c.rows(0), c.rows(1 + b)))
        q = R.bf16(c.rng.standard_normal((n, hq, d)))
        _, z, _, size = R.attention(q, k, v, prompt, d ** -0.5)
        z = z.astype(np.float32)
        c.kv.set_block_table(table[b:b + 1])
        c.kv.attn_mass(rows_to_dev(q), torch.from_numpy(z).cuda(), [prompt], [n], mass)
        got = R.mass(q, z, k, prompt, d ** -0.5)
        pos = np.arange(prompt + n)
        page, slot = table[b][pos // PAGE], pos % PAGE
        old = np.where(pos < prompt, want[page, :, slot].T, 0.0).T
        want[page, :, slot] = old + got
        # as in test_gpu_evict.test_mass; a later call carries what an earlier one left
        rel = 2 * R.score_bound(d, size) + 2.0 ** -22 * np.abs(z).max() + 2.0 ** -21
        kept = np.where(pos < prompt, bound[page, :, slot].T, 0.0).T
        bound[page, :, slot] = kept * (1 + 2.0 ** -24) + got * (rel + 2.0 ** -24 * (n * hq // hkv + 20)) \
            + 2.0 ** -24 * (old + got) + 1e-38
    off = np.abs(host(mass) - want) - bound
    assert off.max() <= 0, off.max()
