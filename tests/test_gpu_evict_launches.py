"""Evictions of more (task, kv head) pairs than one launch takes (needs an MI355X)."""
import numpy as np
import pytest
import torch

import paper_2608_10402_amd as tide

pytestmark = pytest.mark.gpu

PAGE = 16


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("inplace", [True, False])
def test_more_pairs_than_a_launch_takes(bits, inplace):
    """16 tasks of a page each with 65,536 kv heads: 2^20 pairs."""
    n, hkv, d = 16, 65536, 64
    lens = np.array([16 - b % 4 for b in range(n)], np.int32)
    keep = np.array([1 + b % 9 for b in range(n)], np.int32)
    gen = torch.Generator(device="cuda").manual_seed(5)
    table = np.random.default_rng(1).permutation(n).astype(np.int32)[:, None]
    pages = n if inplace else 2 * n
    kv = (tide.PagedKV4 if bits == 4 else tide.PagedKV)(pages, hkv, hkv, d, table, fill_canary=False)
    new = None if inplace else torch.arange(n, 2 * n, dtype=torch.int32, device="cuda")[:, None].contiguous()
    for x in ([kv.pool] if bits == 4 else [kv.k_pool, kv.v_pool]):
        for page in range(pages):  # bytes of any value; the rows are compared as they are
            x[page].view(torch.uint8).random_(0, 256, generator=gen)
    mass = torch.rand((pages, hkv, PAGE), generator=gen, device="cuda")
    mass0 = mass.clone()

    def rows(page):
        """K and V of a page [Hkv][16][bytes or values of a row]."""
        if bits == 16:
            return kv.k_pool[page].view(torch.int16).clone(), kv.v_pool[page].view(torch.int16).clone()
        old, kv.block_table = kv.block_table, torch.full((1, 1), page, dtype=torch.int32, device="cuda")
        got = kv.unpack([0], [PAGE])
        kv.block_table = old
        return tuple(x.view(torch.int16).transpose(0, 1).contiguous() for x in got)

    before = {int(p): rows(int(p)) for p in (table[0, 0], table[7, 0], table[15, 0])}
    kept = kv.evict(mass, lens, keep, new_block_table=new)
    at = 0
    for b in range(n):
        page, k = int(table[b, 0]), int(keep[b])
        order = torch.sort(mass0[page, :, : int(lens[b])], dim=1, descending=True, stable=True).indices[:, :k]
        idx = order.sort(1).values  # [Hkv][keep]
        assert torch.equal(kept[at: at + k].t().long(), idx), b
        to = page if inplace else n + b
        want = mass0[to].clone()
        want[:, :k] = mass0[page].gather(1, idx)
        assert torch.equal(mass[to], want), b
        if page in before:
            for x, y in zip(before[page], rows(to)):
                assert torch.equal(y[:, :k], x.gather(1, idx[..., None].expand(-1, -1, d))), b
        at += k
