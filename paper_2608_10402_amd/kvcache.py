"""Paged KV pools on one device with the entry points bound to them: `PagedKV` holds K and V in
bf16, `PagedKV4` in 4 bits.  `PageTable` is a block table whose lengths and free pages live on the
device too.

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
        self._rows_ws, self._rows_replaced, self._rows_fit = None, [], {}
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


    # ---- steps whose rows, lengths and block lists are device data.  They have a workspace of their own.  A graph goes on
    # using the one that it was captured with, so one that a larger call replaces lives as long as this object.  What is
    # in flight at once (a replay, and a call on another stream) takes a PagedKV each over the same pools.

    def _rows_workspace(self, op, rows, longest=0):
        """A workspace for a call of `op` with this many rows and this budget or longest context, and for every
        smaller one."""
        fit = self._rows_fit.get(op, (-1, 0))
        if rows > fit[0] or longest > fit[1]:
            fit = max(rows, fit[0]), max(longest, fit[1])
            need = _lib.tide_rows_workspace_bound(op, fit[0], self.dims, budget=fit[1], max_len=fit[1])
            old = self._rows_ws
            if old is None or old.numel() < need:
                # (at least twice the last: all that were replaced take less than the present one)
                size = max(need, 1 << 16 if old is None else 2 * old.numel())
                self._rows_ws = _lib.alloc_workspace(size, self.device)
                if old is not None:
                    self._rows_replaced.append(old)
            self._rows_fit[op] = fit
        return self._rows_ws

    def new_bounds(self):
        """Key bounds for append_slots, key_bounds and select_blocks: (bounds, units) of every page."""
        shape = (self.num_pages, self.dims.num_kv_heads, 2, self.dims.head_dim)
        return (torch.zeros(shape, dtype=torch.int8, device=self.device),
                torch.zeros(shape[:2], dtype=torch.int8, device=self.device))

    def append_slots(self, k_new, v_new, row_slot, bounds=None, stream=None):
        """Store the rows' K/V in their slots (tide_slot_append); with bounds, bring those of the
        pages that change up to date."""
        b, u = bounds if bounds is not None else (None, None)
        _lib.tide_slot_append(k_new, v_new, row_slot, self.k_pool, self.v_pool, self.dims, b, u,
                              self._rows_workspace(_lib.TIDE_OP_SLOT_APPEND, 0), stream)

    def key_bounds(self, lens, bounds, from_lens=None, max_len: int = 0, stream=None):
        """Key bounds of the pages that hold positions from_lens (None: 0) .. lens - 1 of each task, both on
        the device (tide_key_bounds): after append, extend_append, evict and what else writes keys, and, with
        from_lens = lens - 1, after a PageTable.map that cut contexts inside a page."""
        _lib.tide_key_bounds(self.k_pool, self.block_table, lens, bounds[0], bounds[1], self.dims, from_lens, max_len,
                             self._rows_workspace(_lib.TIDE_OP_KEY_BOUNDS, 0), stream)
        return bounds

    def select_blocks(self, q, row_task, row_pos, bounds, budget: int, sink: int = 0, recent: int = 0,
                      max_len: int = 0, out=None, stream=None):
        """The `budget` blocks that each row and kv head attends to (tide_block_select), int32
        [rows][Hkv][budget]; those of padding rows are not written."""
        if out is None:
            out = torch.empty((q.shape[0], self.dims.num_kv_heads, budget), dtype=torch.int32, device=q.device)
        longest = min(self.block_table.shape[1] * self.dims.page_size, 2**31 - 1)
        longest = min(max_len, longest) if max_len > 0 else longest
        ws = self._rows_workspace(_lib.TIDE_OP_BLOCK_SELECT, q.shape[0], longest)
        _lib.tide_block_select(q, row_task, row_pos, bounds[0], bounds[1], self.block_table, budget, self.dims, out,
                               sink, recent, max_len, ws, stream)
        return out

    def sparse(self, q, row_task, row_pos, sel, out=None, lse=None, stream=None):
        """Attention of each row over the blocks in sel (tide_sparse_attn); padding rows are not
        written."""
        out = torch.empty_like(q) if out is None else out
        ws = self._rows_workspace(_lib.TIDE_OP_SPARSE_ATTN, q.shape[0], sel.shape[-1])
        _lib.tide_sparse_attn(q, self.k_pool, self.v_pool, self.block_table, row_task, row_pos, sel, self.dims, out, lse,
                              ws, stream)
        return out


class PageTable:
    """Block table, lengths and free pages of num_tasks tasks on the device, changed by `map` alone, so
    that a step (captured or not) needs no lengths from the host.  pages: how many there are, or the
    ids that are free.  Use `block_table` as a PagedKV's: `kv.block_table = table.block_table`."""

    def __init__(self, num_tasks: int, pages_per_task: int, pages, device="cuda"):
        self.device = torch.device(device)
        # the lowest ids on top of the stack
        ids = np.arange(pages)[::-1] if np.ndim(pages) == 0 else np.asarray(pages)
        self.free_pages = torch.from_numpy(np.ascontiguousarray(ids, dtype=np.int32)).to(self.device)
        self.free_count = torch.full((1,), self.free_pages.numel(), dtype=torch.int32, device=self.device)
        self.block_table = torch.zeros((num_tasks, pages_per_task), dtype=torch.int32, device=self.device)
        self.lens = torch.zeros(num_tasks, dtype=torch.int32, device=self.device)
        self.row_start = torch.zeros(num_tasks + 1, dtype=torch.int32, device=self.device)
        self._dims = _lib.make_dims(1, 1, 64, 1.0)  # (the page size)

    def new_rows(self, num_rows: int):
        """(row_task, row_pos, row_slot) for `map`, all padding."""
        return (torch.full((num_rows,), -1, dtype=torch.int32, device=self.device),
                torch.full((num_rows,), -1, dtype=torch.int32, device=self.device),
                torch.full((num_rows,), -1, dtype=torch.int64, device=self.device))

    def map(self, want_lens, rows, stream=None):
        """Bring every task's length to want_lens (device int32 [num_tasks]), taking pages or giving them
        back (tide_page_map), and put the new tokens into rows (from new_rows).  A task that is refused
        keeps its length: lens != want_lens.  One that is cut inside a page leaves that page its key bounds
        until the next append to it: PagedKV.key_bounds(lens, bounds, from_lens=lens - 1) renews them."""
        _lib.tide_page_map(self.lens, want_lens, self.block_table, self.free_pages, self.free_count, self.lens,
                           self.free_count, self.row_start, rows[0], rows[1], rows[2], self._dims, stream)
        return rows


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
