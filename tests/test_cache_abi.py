"""Refusals of the 4-bit cache, attention mass and eviction, and the plans behind them, on the CPU:
every call here fails its checks (or is a no-op) before any device work."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2608_10402_amd as tide
from paper_2608_10402_amd import _lib
from test_codegen import _asm, loops_with_scratch

GOOD = _lib.make_dims(28, 4, 128, 1 / math.sqrt(128))
BAD = [(_lib.make_dims(8, 2, 96, 0.1), tide.TIDE_ERR_UNSUPPORTED), (_lib.make_dims(34, 2, 64, 0.1), tide.TIDE_ERR_UNSUPPORTED),
       (_lib.make_dims(8, 2, 64, 0.1, page_size=32), tide.TIDE_ERR_UNSUPPORTED),
       (_lib.make_dims(8, 2, 64, float("nan")), tide.TIDE_ERR_INVALID_ARG), (None, tide.TIDE_ERR_INVALID_ARG)]
X = 1 << 20  # an aligned address that nothing reads: the calls fail first

# entry point: its arguments in order, with lengths that are right
CALLS = {
    "tide_kv4_append": dict(k_new=X, v_new=X, pool=X, pages=10, bt=X, stride=4, n=1, prefix=[3], extend=[2], dims=GOOD,
                            ws=X, ws_bytes=1 << 20, stream=None),
    "tide_kv4_unpack": dict(pool=X, pages=10, bt=X, stride=4, n=1, prefix=[3], extend=[2], dims=GOOD, k_out=X, v_out=X,
                            ws=X, ws_bytes=1 << 20, stream=None),
    "tide_kv4_decode_attn": dict(q=X, pool=X, pages=10, bt=X, stride=4, n=1, kv=[5], dims=GOOD, out=X, lse=None, ws=X,
                                 ws_bytes=1 << 20, stream=None),
    "tide_kv4_decode_append_attn": dict(q=X, k_new=X, v_new=X, pool=X, pages=10, bt=X, stride=4, n=1, kv=[5], dims=GOOD,
                                        out=X, lse=None, ws=X, ws_bytes=1 << 20, stream=None),
    "tide_kv4_extend_attn": dict(q=X, pool=X, pages=10, bt=X, stride=4, n=1, prefix=[3], extend=[2], dims=GOOD, out=X,
                                 lse=None, ws=X, ws_bytes=1 << 20, stream=None),
    "tide_attn_mass": dict(q=X, lse_in=X, pool=X, pages=10, bt=X, stride=4, n=1, prefix=[3], extend=[2], counted=None,
                           dims=GOOD, mass=X, ws=X, ws_bytes=1 << 20, stream=None),
    "tide_kv4_attn_mass": dict(q=X, lse_in=X, pool=X, pages=10, bt=X, stride=4, n=1, prefix=[3], extend=[2], counted=None,
                               dims=GOOD, mass=X, ws=X, ws_bytes=1 << 20, stream=None),
    "tide_kv_evict": dict(k_pool=X, v_pool=X, mass=X, pages=10, bt=X, stride=4, new=None, new_stride=0, n=1, kv=[5],
                          keep=[3], recent=None, dims=GOOD, kept=None, ws=X, ws_bytes=1 << 20, stream=None),
    "tide_kv4_evict": dict(pool=X, mass=X, pages=10, bt=X, stride=4, new=None, new_stride=0, n=1, kv=[5], keep=[3],
                           recent=None, dims=GOOD, kept=None, ws=X, ws_bytes=1 << 20, stream=None),
}


def call(name, **over):
    args = dict(CALLS[name])
    for k in over:
        assert k in args, (name, k)
    args.update(over)
    hold, out = [], []
    for v in args.values():
        if isinstance(v, list):
            hold.append(np.ascontiguousarray(v, np.int32))
            out.append(hold[-1].ctypes.data)
        elif isinstance(v, _lib.tide_dims):
            out.append(ctypes.byref(v))
        else:
            out.append(v)
    return getattr(tide.load(), name)(*out)


POINTERS = [(n, k) for n, a in CALLS.items() for k in a
            if k in ("k_new", "v_new", "pool", "bt", "k_out", "v_out", "q", "out", "lse_in", "mass", "k_pool", "v_pool", "ws")]


@pytest.mark.parametrize("name,arg", POINTERS)
def test_null_pointers(name, arg):
    assert call(name, **{arg: None}) == tide.TIDE_ERR_INVALID_ARG


@pytest.mark.parametrize("name,arg", [p for p in POINTERS if p[1] not in ("bt", "lse_in")])
def test_pointers_off_16_bytes(name, arg):
    assert call(name, **{arg: X + 8}) == tide.TIDE_ERR_INVALID_ARG


@pytest.mark.parametrize("name", CALLS)
def test_shapes_and_counts(name):
    for dims, code in BAD:
        assert call(name, dims=dims) == code
    assert call(name, n=-1) == tide.TIDE_ERR_INVALID_ARG
    assert call(name, n=0) == tide.TIDE_OK
    assert call(name, pages=0) == tide.TIDE_ERR_INVALID_ARG
    assert call(name, stride=0) == tide.TIDE_ERR_INVALID_ARG
    assert call(name, ws_bytes=64) == tide.TIDE_ERR_CAPACITY


@pytest.mark.parametrize("name", [n for n, a in CALLS.items() if "extend" in a])
def test_extend_lengths(name):
    assert call(name, prefix=[-1]) == tide.TIDE_ERR_INVALID_ARG
    assert call(name, extend=[-1]) == tide.TIDE_ERR_INVALID_ARG
    assert call(name, prefix=None) == tide.TIDE_ERR_INVALID_ARG
    assert call(name, extend=None) == tide.TIDE_ERR_INVALID_ARG
    assert call(name, prefix=[2**31 - 5], extend=[10]) == tide.TIDE_ERR_INVALID_ARG
    assert call(name, prefix=[60], extend=[5]) == tide.TIDE_ERR_CAPACITY
    assert call(name, extend=[0]) == tide.TIDE_OK
    if "mass" in name:
        for c in ([-1], [6]):
            assert call(name, counted=c) == tide.TIDE_ERR_INVALID_ARG


@pytest.mark.parametrize("name", ["tide_kv4_decode_attn", "tide_kv4_decode_append_attn"])
def test_decode_lengths(name):
    assert call(name, kv=[0]) == tide.TIDE_ERR_INVALID_ARG
    assert call(name, kv=None) == tide.TIDE_ERR_INVALID_ARG
    assert call(name, kv=[65]) == tide.TIDE_ERR_CAPACITY


@pytest.mark.parametrize("name", ["tide_kv_evict", "tide_kv4_evict"])
def test_evict_lengths(name):
    assert call(name, keep=[6]) == tide.TIDE_ERR_INVALID_ARG
    assert call(name, keep=[-1]) == tide.TIDE_ERR_INVALID_ARG
    assert call(name, kv=[-1], keep=[0]) == tide.TIDE_ERR_INVALID_ARG
    assert call(name, recent=[4]) == tide.TIDE_ERR_INVALID_ARG
    assert call(name, recent=[-1]) == tide.TIDE_ERR_INVALID_ARG
    assert call(name, kv=None) == tide.TIDE_ERR_INVALID_ARG
    assert call(name, kv=[65]) == tide.TIDE_ERR_CAPACITY
    assert call(name, new=X, new_stride=0) == tide.TIDE_ERR_INVALID_ARG
    assert call(name, kv=[40], keep=[33], new=X, new_stride=2) == tide.TIDE_ERR_CAPACITY
    assert call(name, keep=[0]) == tide.TIDE_OK


def size(op, a, b=None, dims=GOOD):
    return tide.tide_workspace_size(op, a, b, dims)


def test_workspace_sizes():
    assert 0 < size(tide.TIDE_OP_KV4_APPEND, [3], [5]) <= size(tide.TIDE_OP_KV_APPEND, [3], [5])
    assert size(tide.TIDE_OP_KV4_EXTEND, [5000], [4]) < 1 << 22                 # the codes themselves
    staged = size(tide.TIDE_OP_KV4_EXTEND, [5000], [500])
    assert staged > 5500 * 4 * 128 * 4                                         # K and V of the task in bf16
    many = size(tide.TIDE_OP_KV4_EXTEND, [5000] * 100, [500] * 100)
    assert (1 << 29) < many < (1 << 30) + (1 << 28)                            # rounds of at most 1 GiB
    one = size(tide.TIDE_OP_KV4_EXTEND, [700000], [500])
    assert one > 700500 * 4 * 128 * 4                                          # but a whole task at least
    assert size(tide.TIDE_OP_KV_EVICT, [100], [50]) < size(tide.TIDE_OP_KV_EVICT, [1000], [900])
    for op in (tide.TIDE_OP_KV4_APPEND, tide.TIDE_OP_KV4_UNPACK, tide.TIDE_OP_KV4_EXTEND, tide.TIDE_OP_ATTN_MASS,
               tide.TIDE_OP_KV_EVICT):
        assert size(op, [], []) > 0
    with pytest.raises(tide.TideError):
        size(tide.TIDE_OP_KV_EVICT, [10], [11])


def test_longest_eviction():
    most = 0x7FF00000  # TIDE_EVICT_MAX_LEN
    assert size(tide.TIDE_OP_KV_EVICT, [most], [5]) > 0
    with pytest.raises(tide.TideError):
        size(tide.TIDE_OP_KV_EVICT, [most + 1], [5])


def test_plan_info_of_the_4_bit_attention():
    info = tide.tide_plan_info_get(tide.TIDE_OP_KV4_DECODE, [100, 2000], None, GOOD)
    assert info["num_items"] % 4 == 0 and info["run_steps"] >= 1
    few = tide.tide_plan_info_get(tide.TIDE_OP_KV4_EXTEND, [100, 2000], [3, 1], GOOD)
    assert few["run_steps"] >= 1
    more = tide.tide_plan_info_get(tide.TIDE_OP_KV4_EXTEND, [100, 2000], [300, 1], GOOD)
    assert more["run_steps"] == 0 and more["num_items"] > 0


class TestBinding:
    """What the Python layer refuses by itself (host tensors; no call reaches the library)."""

    def test_pool_shape(self):
        t = torch.zeros((3, 4, 100), dtype=torch.uint8)
        with pytest.raises(ValueError, match="kv4_pool"):
            tide.tide_kv4_decode_attn(None, t, None, [1], GOOD, None)

    def test_device_and_types(self):
        pool = torch.zeros((3, 4, 17 * 128), dtype=torch.uint8)
        bt = torch.zeros((1, 3), dtype=torch.int32)
        q = torch.zeros((1, 28, 128), dtype=torch.bfloat16)
        with pytest.raises(ValueError, match="device"):
            tide.tide_kv4_decode_attn(q, pool, bt, [1], GOOD, q.clone())
        with pytest.raises(ValueError, match="shape"):
            tide.tide_kv4_decode_attn(q[:, :27], pool, bt, [1], GOOD, q)
        with pytest.raises(ValueError, match="counted_lens"):
            tide.tide_kv4_attn_mass(q, torch.zeros(1, 28), pool, bt, [0], [1], GOOD, torch.zeros(3, 4, 16), [0, 0])
        with pytest.raises(ValueError, match="mass"):
            tide.tide_kv4_evict(pool, torch.zeros(3, 4, 8), bt, [1], [1], GOOD)
        with pytest.raises(ValueError, match="kept"):
            tide.tide_kv4_evict(pool, torch.zeros(3, 4, 16), bt, [9], [5], GOOD, kept=torch.zeros((4, 4), dtype=torch.int32))
        with pytest.raises(ValueError, match="one entry per task"):
            tide.tide_kv4_evict(pool, torch.zeros(3, 4, 16), bt, [9], [5, 5], GOOD)

    def test_pool_argument(self):
        with pytest.raises(ValueError, match="pool"):
            tide.PagedKV4(2, 8, 2, 64, [[0, 1]], device="cpu", pool=torch.zeros((2, 2, 17), dtype=torch.uint8))
        kv = tide.PagedKV4(2, 8, 2, 64, [[0, 1]], device="cpu")
        assert tuple(kv.pool.shape) == (2, 2, tide.kv4_block_bytes(64)) and (kv.pool == 255).all()
        assert tuple(kv.new_mass().shape) == (2, 2, 16)


@pytest.mark.parametrize("src", ["kv4_store.hip", "kv4_decode.hip", "attn_mass.hip", "kv_evict.hip"])
def test_no_scratch_access_inside_loops(tmp_path, src):
    found = loops_with_scratch(_asm(tmp_path, src))
    assert found
    bad = [x for x in found if x[2]]
    assert not bad, bad
