"""Streams of the calls whose rows and lengths are device data (needs an MI355X).

Inputs are written on a side stream behind a bounded spin kernel, and the calls follow on it, or on another that
waits for it.  A call that went to any other stream would run at once, with the old inputs or the old rows."""
import time

import numpy as np
import pytest
import torch

from test_gpu_rows import BUDGET, D, HKV, HQ, RECENT, SINK, dev, engine, normal

pytestmark = pytest.mark.gpu

SPIN = 50_000_000  # tens of ms
FIRST, NEXT = [30, 100, 5], [31, 160, 6]


class Step:
    """A step's inputs in buffers that are written late, and all that it works on."""

    def __init__(self, seed):
        rng = np.random.default_rng(seed)
        self.kv, self.table, self.bounds = engine(3, 20, 60)
        self.rows = self.table.new_rows(sum(NEXT) - sum(FIRST) + 2)
        n = self.rows[0].numel()
        prompt = [normal(rng, sum(FIRST), x, D) for x in (HKV, HKV)]
        rows = self.table.new_rows(sum(FIRST))
        self.table.map(dev(FIRST), rows)
        self.kv.append_slots(*prompt, rows[2], self.bounds)
        self.late = [dev(NEXT)] + [normal(rng, n, x, D) for x in (HQ, HKV, HKV)]
        self.early = [dev(FIRST)] + [normal(rng, n, x, D) for x in (HQ, HKV, HKV)]
        self.sel = torch.full((n, HKV, BUDGET), -5, dtype=torch.int32, device="cuda")
        self.out = torch.zeros((n, HQ, D), dtype=torch.bfloat16, device="cuda")
        self.lse = torch.zeros((n, HQ), device="cuda")
        self.fresh = self.kv.new_bounds()

    def write(self):
        for a, b in zip(self.early, self.late):
            a.copy_(b)

    def calls(self, stream=None):
        want, q, k, v = self.early
        self.table.map(want, self.rows, stream=stream)
        self.kv.append_slots(k, v, self.rows[2], self.bounds, stream=stream)
        self.kv.key_bounds(self.table.lens, self.fresh, stream=stream)
        self.kv.select_blocks(q, *self.rows[:2], self.bounds, BUDGET, SINK, RECENT, out=self.sel, stream=stream)
        self.kv.sparse(q, *self.rows[:2], self.sel, out=self.out, lse=self.lse, stream=stream)

    def results(self):
        return [self.table.lens, self.table.block_table, *self.rows, self.kv.k_pool.view(torch.int16),
                self.kv.v_pool.view(torch.int16), *self.bounds, *self.fresh, self.sel, self.out, self.lse]


def alone(seed):
    s = Step(seed)
    s.write()
    torch.cuda.synchronize()
    s.calls()
    torch.cuda.synchronize()
    assert s.table.lens.tolist() == NEXT
    return s.results()


def stream_beside_the_default():
    """A stream whose work the default one does not wait for, as it does where the two share a hardware queue (any
    stream, if there is none)."""
    for _ in range(8):
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        start = time.perf_counter()
        with torch.cuda.stream(side):
            torch.cuda._sleep(SPIN // 4)
        torch.zeros(16, device="cuda")
        torch.cuda.current_stream().synchronize()
        beside = time.perf_counter() - start
        side.synchronize()
        if beside < (time.perf_counter() - start) / 2:
            break
    return side


@pytest.mark.parametrize("how", ["current", "argument", "handle"])
def test_calls_go_to_their_stream(how):
    want = alone(51)
    s, side = Step(51), stream_beside_the_default()
    # (padding rows: the workspaces are there, and nothing below allocates)
    s.kv.select_blocks(s.early[1], *s.rows[:2], s.bounds, BUDGET, out=s.sel)
    s.kv.sparse(s.early[1], *s.rows[:2], s.sel, out=s.out)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(SPIN)
        s.write()
        if how == "current":
            s.calls()
    if how != "current":
        s.calls(side if how == "argument" else side.cuda_stream)
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(s.results(), want)):
        assert torch.equal(a, b), i


def test_two_engines_behind_spins_of_their_own():
    """The second engine's stream spins longer; each step's calls take turns, and neither waits for the other."""
    want = [alone(52), alone(53)]
    steps, streams = [Step(52), Step(53)], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for s, stream, spin in zip(steps, streams, (SPIN // 4, SPIN)):
        with torch.cuda.stream(stream):
            torch.cuda._sleep(spin)
            s.write()
    for s, stream in zip(steps, streams):
        with torch.cuda.stream(stream):
            s.calls()
    streams[0].synchronize()
    first = [x.cpu() for x in steps[0].results()]
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(first, want[0])):
        assert torch.equal(a, b.cpu()), i
    for i, (a, b) in enumerate(zip(steps[1].results(), want[1])):
        assert torch.equal(a, b), i


def test_a_step_over_two_streams():
    """A page map on one stream and the rest on another that waits for its event."""
    want = alone(54)
    s, a, b = Step(54), torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(a):
        torch.cuda._sleep(SPIN)
        s.write()
        s.table.map(s.early[0], s.rows)
        mapped = a.record_event()
    with torch.cuda.stream(b):
        b.wait_event(mapped)
        _, q, k, v = s.early
        s.kv.append_slots(k, v, s.rows[2], s.bounds)
        s.kv.key_bounds(s.table.lens, s.fresh)
        s.kv.select_blocks(q, *s.rows[:2], s.bounds, BUDGET, SINK, RECENT, out=s.sel)
        s.kv.sparse(q, *s.rows[:2], s.sel, out=s.out, lse=s.lse)
    torch.cuda.synchronize()
    for i, (x, y) in enumerate(zip(s.results(), want)):
        assert torch.equal(x, y), i
