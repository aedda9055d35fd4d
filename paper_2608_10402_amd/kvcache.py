"""Paged KV pools on one device with the entry points bound to them: `PagedKV` holds K and V in
bf16, `PagedKV4` in 4 bits.

Convenience layer over the C ABI: owns the page pools, the block table and a
grow-only workspace, and forwards each call to libtide.so.  No arithmetic happens here.
"""
from __future__ import annotations

import math

import numpy as np
import torch

from . import _lib

CANARY_BITS = 0x7FC0  # bf16 quiet NaN; unused pool slots hold it so leaks are visible


class _Paged:
    """What the pools share: dims, the block table and the workspace."""

    def __init__(self, num_q_heads, num_kv_heads, head_dim, block_table, sm_scale, device):
        self.device = torch.device(device)
        self.dims = _lib.make_dims(num_q_heads, num_kv_heads, head_dim,
                                   sm_scale if sm_scale is not None else 1.0 / math.sqrt(head_dim))
        self.set_block_table(block_table)
        self._ws = None

    @property
    def num_q_heads(self):
        return self.dims.num_q_heads

    @property
    def head_dim(self):
        return self.dims.head_dim

    def set_block_table(self, block_table):
        bt = torch.as_tensor(np.ascontiguousarray(block_table, dtype=np.int32))
        self.block_table = bt.to(self.device).contiguous()

    def workspace(self, nbytes: int) -> torch.Tensor:
        if self._ws is None or self._ws.numel() < nbytes:
            self._ws = _lib.alloc_workspace(max(nbytes, 1 << 16), self.device)
        return self._ws

    def _call(self, size, call):
        """call(workspace), with a workspace that is large enough.  The library plans every
        call and refuses a workspace too small for it before any device work, so a call is
        planned once as a rule, and its size asked for only then."""
        if self._ws is None:
            self.workspace(size())
        try:
            call(self._ws)
        except _lib.TideError as e:
            if e.status != _lib.TIDE_ERR_CAPACITY:
                raise
            need = size()
            if need <= self._ws.numel():  # the block table's capacity, not the workspace's
                raise
            call(self.workspace(need))

    def new_mass(self) -> torch.Tensor:
        """Sums for attn_mass and evict, one per pool slot and kv head, all zero."""
        return torch.zeros((self.num_pages, self.dims.num_kv_heads, self.dims.page_size),
                           dtype=torch.float32, device=self.device)

    def _evict(self, entry, mass, kv_lens, keep_lens, recent_lens, new_block_table, kept, stream):
        if kept is None:
            kept = torch.empty((_lib.rows_of(keep_lens), self.dims.num_kv_heads), dtype=torch.int32,
                               device=self.device)
        self._call(lambda: _lib.tide_workspace_size(_lib.TIDE_OP_KV_EVICT, kv_lens, keep_lens,
                                                    self.dims),
                   lambda ws: entry(mass, self.block_table, kv_lens, keep_lens, self.dims,
                                    recent_lens, new_block_table, kept, ws, stream))
        return kept


class PagedKV(_Paged):
    def __init__(self, num_pages: int, num_q_heads: int, num_kv_heads: int, head_dim: int,
                 block_table, sm_scale: float | None = None, device="cuda",
                 fill_canary: bool = True):
        super().__init__(num_q_heads, num_kv_heads, head_dim, block_table, sm_scale, device)
        shape_k = shape_v = (num_pages, num_kv_heads, 16, head_dim)
        if fill_canary:
            self.k_pool = torch.full(shape_k, CANARY_BITS, dtype=torch.int16,
                                     device=self.device).view(torch.bfloat16)
            self.v_pool = torch.full(shape_v, CANARY_BITS, dtype=torch.int16,
                                     device=self.device).view(torch.bfloat16)
        else:
            self.k_pool = torch.empty(shape_k, dtype=torch.bfloat16, device=self.device)
            self.v_pool = torch.empty(shape_v, dtype=torch.bfloat16, device=self.device)

    @property
    def num_pages(self):
        return self.k_pool.shape[0]

    def append(self, k_new, v_new, prefix_lens, extend_lens, stream=None):
        self._call(lambda: _lib.tide_workspace_size(_lib.TIDE_OP_KV_APPEND, prefix_lens,
                                                    extend_lens, self.dims),
                   lambda ws: _lib.tide_kv_append(k_new, v_new, self.k_pool, self.v_pool,
                                                  self.block_table, prefix_lens, extend_lens,
                                                  self.dims, ws, stream))

    def extend(self, q, prefix_lens, extend_lens, out=None, lse=None, stream=None):
        out = torch.empty_like(q) if out is None else out
        self._call(lambda: _lib.tide_workspace_size(_lib.TIDE_OP_EXTEND, prefix_lens, extend_lens,
                                                    self.dims),
                   lambda ws: _lib.tide_extend_attn(q, self.k_pool, self.v_pool, self.block_table,
                                                    prefix_lens, extend_lens, self.dims, out, lse,
                                                    ws, stream))
        return out

    def extend_append(self, q, k_new, v_new, prefix_lens, extend_lens, out=None, lse=None,
                      stream=None):
        """Append the new tokens' K/V and run extend attention, fused in one call."""
        out = torch.empty_like(q) if out is None else out
        self._call(lambda: _lib.tide_workspace_size(_lib.TIDE_OP_EXTEND, prefix_lens, extend_lens,
                                                    self.dims),
                   lambda ws: _lib.tide_extend_append_attn(q, k_new, v_new, self.k_pool,
                                                           self.v_pool, self.block_table,
                                                           prefix_lens, extend_lens, self.dims,
                                                           out, lse, ws, stream))
        return out

    def decode(self, q, kv_lens, num_splits: int = 0, out=None, lse=None, stream=None):
        out = torch.empty_like(q) if out is None else out
        self._call(lambda: _lib.tide_workspace_size(_lib.TIDE_OP_DECODE, kv_lens, None, self.dims,
                                                    num_splits),
                   lambda ws: _lib.tide_decode_attn(q, self.k_pool, self.v_pool, self.block_table,
                                                    kv_lens, self.dims, out, lse, num_splits, ws,
                                                    stream))
        return out

    def decode_append(self, q, k_new, v_new, kv_lens, num_splits: int = 0, out=None, lse=None,
                      stream=None):
        """Append each task's newest token (position kv_lens - 1) and decode, fused."""
        out = torch.empty_like(q) if out is None else out
        self._call(lambda: _lib.tide_workspace_size(_lib.TIDE_OP_DECODE, kv_lens, None, self.dims,
                                                    num_splits),
                   lambda ws: _lib.tide_decode_append_attn(q, k_new, v_new, self.k_pool,
                                                           self.v_pool, self.block_table, kv_lens,
                                                           self.dims, out, lse, num_splits, ws,
                                                           stream))
        return out

    def decode_noalloc(self, q, kv_lens, num_splits: int = 0, out=None, lse=None, stream=None):
        """Decode in the library's static device scratch: no workspace is allocated."""
        out = torch.empty_like(q) if out is None else out
        _lib.tide_decode_attn_noalloc(q, self.k_pool, self.v_pool, self.block_table, kv_lens,
                                      self.dims, out, lse, num_splits, stream)
        return out

    def decode_shared(self, q, kv_lens, group_start, shared_lens, num_splits: int = 0, out=None,
                      lse=None, stream=None):
        out = torch.empty_like(q) if out is None else out
        self._call(lambda: _lib.tide_workspace_size_shared(kv_lens, group_start, shared_lens,
                                                           self.dims, num_splits),
                   lambda ws: _lib.tide_decode_attn_shared(q, self.k_pool, self.v_pool,
                                                           self.block_table, kv_lens, group_start,
                                                           shared_lens, self.dims, out, lse,
                                                           num_splits, ws, stream))
        return out

    def prefill(self, q, seq_lens, out=None, lse=None, stream=None):
        out = torch.empty_like(q) if out is None else out
        self._call(lambda: _lib.tide_workspace_size(_lib.TIDE_OP_FULL_PREFILL, seq_lens, None,
                                                    self.dims),
                   lambda ws: _lib.tide_full_prefill_attn(q, self.k_pool, self.v_pool,
                                                          self.block_table, seq_lens, self.dims,
                                                          out, lse, ws, stream))
        return out

    def attn_mass(self, q, lse, prefix_lens, extend_lens, mass, counted_lens=None, stream=None):
        """Add the attention weights of the new tokens' rows to the keys' sums (tide_attn_mass).
        Tasks that share pages go into calls of their own."""
        self._call(lambda: _lib.tide_workspace_size(_lib.TIDE_OP_ATTN_MASS, prefix_lens, extend_lens,
                                                    self.dims),
                   lambda ws: _lib.tide_attn_mass(q, lse, self.k_pool, self.block_table, prefix_lens,
                                                  extend_lens, self.dims, mass, counted_lens, ws,
                                                  stream))
        return mass

    def evict(self, mass, kv_lens, keep_lens, recent_lens=None, new_block_table=None, kept=None,
              stream=None):
        """Keep each task's recent and heaviest positions (tide_kv_evict); returns the kept
        positions [sum of keep_lens][Hkv].  With a new_block_table the kept positions lie in its
        pages: make it the block table (`block_table = ...`) to go on with them."""
        return self._evict(lambda *a: _lib.tide_kv_evict(self.k_pool, self.v_pool, *a), mass, kv_lens,
                           keep_lens, recent_lens, new_block_table, kept, stream)


class PagedKV4(_Paged):
    """A pool that holds K and V in 4 bits: blocks of 32 codes (e2m1) with a power of two each, 17/64
    of the bf16 pool's bytes (include/tide.h has the format).  pool: an existing uint8 tensor
    [num_pages][Hkv][17 d] to work in."""

    def __init__(self, num_pages: int, num_q_heads: int, num_kv_heads: int, head_dim: int,
                 block_table, sm_scale: float | None = None, device="cuda",
                 fill_canary: bool = True, pool=None):
        super().__init__(num_q_heads, num_kv_heads, head_dim, block_table, sm_scale, device)
        shape = (num_pages, num_kv_heads, _lib.kv4_block_bytes(head_dim))
        if pool is not None:
            if tuple(pool.shape) != shape:
                raise ValueError("pool must have shape %s, got %s" % (shape, tuple(pool.shape)))
            self.pool = pool
        else:
            self.pool = torch.empty(shape, dtype=torch.uint8, device=self.device)
            if fill_canary:
                self.pool.fill_(255)  # scale bytes of 255: every slot reads as NaN

    @property
    def num_pages(self):
        return self.pool.shape[0]

    def _size(self, op, a, b=None):
        return lambda: _lib.tide_workspace_size(op, a, b, self.dims)

    def append(self, k_new, v_new, prefix_lens, extend_lens, stream=None):
        self._call(self._size(_lib.TIDE_OP_KV4_APPEND, prefix_lens, extend_lens),
                   lambda ws: _lib.tide_kv4_append(k_new, v_new, self.pool, self.block_table,
                                                   prefix_lens, extend_lens, self.dims, ws, stream))

    def unpack(self, prefix_lens, extend_lens, k_out=None, v_out=None, stream=None):
        """The values at positions prefix .. prefix + extend - 1 as bf16 rows (K, V)."""
        got = []
        self._call(self._size(_lib.TIDE_OP_KV4_UNPACK, prefix_lens, extend_lens),
                   lambda ws: got.extend(_lib.tide_kv4_unpack(
                       self.pool, self.block_table, prefix_lens, extend_lens, self.dims, k_out,
                       v_out, ws, stream)))
        return tuple(got)

    def decode(self, q, kv_lens, out=None, lse=None, stream=None):
        out = torch.empty_like(q) if out is None else out
        self._call(self._size(_lib.TIDE_OP_KV4_DECODE, kv_lens),
                   lambda ws: _lib.tide_kv4_decode_attn(q, self.pool, self.block_table, kv_lens,
                                                        self.dims, out, lse, ws, stream))
        return out

    def decode_append(self, q, k_new, v_new, kv_lens, out=None, lse=None, stream=None):
        """Append each task's newest token (position kv_lens - 1) and decode, fused."""
        out = torch.empty_like(q) if out is None else out
        self._call(self._size(_lib.TIDE_OP_KV4_DECODE, kv_lens),
                   lambda ws: _lib.tide_kv4_decode_append_attn(q, k_new, v_new, self.pool,
                                                               self.block_table, kv_lens, self.dims,
                                                               out, lse, ws, stream))
        return out

    def extend(self, q, prefix_lens, extend_lens, out=None, lse=None, stream=None):
        """A long extend unpacks the pages of every task of its call into the workspace, which stays
        with the pool object: one among short ones is better off in a call of its own."""
        out = torch.empty_like(q) if out is None else out
        self._call(self._size(_lib.TIDE_OP_KV4_EXTEND, prefix_lens, extend_lens),
                   lambda ws: _lib.tide_kv4_extend_attn(q, self.pool, self.block_table, prefix_lens,
                                                        extend_lens, self.dims, out, lse, ws, stream))
        return out

    def attn_mass(self, q, lse, prefix_lens, extend_lens, mass, counted_lens=None, stream=None):
        """Add the attention weights of the new tokens' rows to the keys' sums (tide_attn_mass).
        Tasks that share pages go into calls of their own."""
        self._call(self._size(_lib.TIDE_OP_ATTN_MASS, prefix_lens, extend_lens),
                   lambda ws: _lib.tide_kv4_attn_mass(q, lse, self.pool, self.block_table, prefix_lens,
                                                      extend_lens, self.dims, mass, counted_lens, ws,
                                                      stream))
        return mass

    def evict(self, mass, kv_lens, keep_lens, recent_lens=None, new_block_table=None, kept=None,
              stream=None):
        """Keep each task's recent and heaviest positions (tide_kv_evict); returns the kept
        positions [sum of keep_lens][Hkv].  With a new_block_table the kept positions lie in its
        pages: make it the block table (`block_table = ...`) to go on with them."""
        return self._evict(lambda *a: _lib.tide_kv4_evict(self.pool, *a), mass, kv_lens, keep_lens,
                           recent_lens, new_block_table, kept, stream)
