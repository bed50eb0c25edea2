"""A cache of 8 or 4 bits a value, over the C ABI (include/tactic.h, tactic_quant_kv): rows
into it and out of it, single-token decode over it, and blocks of it chosen by a cheap score.

As in attention.py, objects hold the workspace and the outputs that their calls return, so
repeated calls allocate nothing; calls of one object must be ordered on one stream.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import torch

from . import _capi as C
from .attention import ScoreMod, _Call, _device, _workspace
from .tactic import RaggedBatch, _indptr

BLOCKS = (16, 32, 64, 128)


class QuantizedCache:
    """The arrays of a quantised cache (see tactic_quant_kv): K, V uint8 [Hkv][total][16 bits] with
    K_scale, V_scale uint8 [Hkv][total][4], or with page_table int32 [B][max_pages] pages
    [num_pages][Hkv][page_size][..]; bounds bf16 [Hkv][total // block + B][2][128] of its blocks of
    `block` rows (total and B those of the batch it is used with)."""

    def __init__(self, K: torch.Tensor, K_scale: torch.Tensor, V: torch.Tensor, V_scale: torch.Tensor,
                 bounds: Optional[torch.Tensor] = None, block: int = 0, page_table: Optional[torch.Tensor] = None):
        if K.shape[-1] not in (64, 128):
            raise ValueError(f"a row of K has 128 bytes (8 bits) or 64 (4 bits), got {K.shape[-1]}")
        if K.dim() != (3 if page_table is None else 4):
            raise ValueError("K must be [Hkv][total][..], with a page table [num_pages][Hkv][page_size][..]")
        if block not in (0,) + BLOCKS:
            raise ValueError("block must be 16, 32, 64 or 128, or 0 without bounds")
        if (bounds is None) != (block == 0):
            raise ValueError("bounds and block go together")
        self.K, self.K_scale, self.V, self.V_scale = K, K_scale, V, V_scale
        self.bounds, self.block, self.page_table = bounds, int(block), page_table
        self.bits = int(K.shape[-1]) // 16

    @staticmethod
    def empty(batch: RaggedBatch, bits: int, block: int = 0) -> "QuantizedCache":
        """A cache for the spans of a batch (its capacities), with bounds of blocks of `block` rows."""
        return QuantizedCache._new(batch, (batch.n_kv_heads, batch.total), bits, block, None)

    @staticmethod
    def empty_pages(batch: RaggedBatch, bits: int, num_pages: int, page_size: int, page_table: torch.Tensor,
                    block: int = 0) -> "QuantizedCache":
        """A cache in pages, for the sequences of a batch."""
        return QuantizedCache._new(batch, (int(num_pages), batch.n_kv_heads, int(page_size)), bits, block, page_table)

    @staticmethod
    def _new(batch, rows, bits, block, page_table):
        if bits not in (8, 4):
            raise ValueError("bits must be 8 or 4")
        if block not in (0,) + BLOCKS:
            raise ValueError("block must be 16, 32, 64 or 128, or 0 without bounds")
        dev = _device(batch)

        def codes(last):
            return torch.zeros(*rows, last, dtype=torch.uint8, device=dev)

        bounds = (torch.zeros(batch.n_kv_heads, batch.total // block + batch.batch, 2, 128, dtype=torch.bfloat16, device=dev)
                  if block else None)
        return QuantizedCache(codes(16 * bits), codes(4), codes(16 * bits), codes(4), bounds, block, page_table)

    def struct(self, call: _Call, batch: RaggedBatch, rows: bool = True) -> C.QuantKV:
        """The C struct after its checks against a batch (rows: its rows are used, not the bounds alone)."""
        t, u8, heads, bits, block = call.tensor, torch.uint8, batch.n_kv_heads, self.bits, self.block
        bounds = None
        if self.bounds is not None:
            bounds = t(self.bounds, "cache.bounds", torch.bfloat16, (heads, batch.total // block + batch.batch, 2, 128))
        if not rows:
            return C.QuantKV(None, None, None, None, bounds, None, bits, block, 0, 0, 0)
        table, pages = self.page_table, (0, 0, 0)
        if table is None:
            wide, scale = (heads, batch.total, 16 * bits), (heads, batch.total, 4)
        else:
            num_pages, _, page_size, _ = self.K.shape
            wide, scale = (num_pages, heads, page_size, 16 * bits), (num_pages, heads, page_size, 4)
            pages = (page_size, table.shape[-1], num_pages)
            table = t(table, "cache.page_table", torch.int32, (batch.batch, pages[1]))
        return C.QuantKV(t(self.K, "cache.K", u8, wide), t(self.K_scale, "cache.K_scale", u8, scale),
                         t(self.V, "cache.V", u8, wide), t(self.V_scale, "cache.V_scale", u8, scale), bounds, table, bits, block,
                         *pages)


class CacheQuantizer:
    """Each sequence's last new_lens[b] rows into a quantised cache (tactic_quant_write) and out of it
    (tactic_quant_read): a prompt, a chunk of one, or a new token.  The lengths are those at the call
    (batch.seq_len), the new rows among them."""

    def __init__(self, batch: RaggedBatch, new_lens: Sequence[int]):
        self.batch, self.new_lens = batch, [int(x) for x in new_lens]
        if len(self.new_lens) != batch.batch:
            raise ValueError("new_lens must name every sequence")
        if any(m < 0 for m in self.new_lens):
            raise ValueError("new_lens must be >= 0")
        self.row_indptr_host = _indptr(self.new_lens)
        self.row_indptr = torch.as_tensor(self.row_indptr_host, device=_device(batch))
        self.total = int(self.row_indptr_host[-1])
        self._shape = batch.struct()
        self._rows = C.QueryShape(self.total, max(self.new_lens), self.row_indptr.data_ptr())
        self._out = None

    def write(self, k: torch.Tensor, v: torch.Tensor, cache: QuantizedCache, stream=None) -> None:
        """k, v bf16 [sum of new_lens][Hkv][128], the sequences' rows one after another; the cache's bounds
        follow if it has them."""
        b = self.batch
        call = _Call(_device(b), stream)
        new = (self.total, b.n_kv_heads, 128)
        kv = cache.struct(call, b)
        call.run("tactic_quant_write", call.tensor(k, "k", torch.bfloat16, new), call.tensor(v, "v", torch.bfloat16, new),
                 ctypes.byref(self._shape), ctypes.byref(self._rows), ctypes.byref(kv))

    def read(self, cache: QuantizedCache, stream=None, K_out: Optional[torch.Tensor] = None,
             V_out: Optional[torch.Tensor] = None):
        """(K, V) bf16 [Hkv][sum of new_lens][128] as the cache holds them (PromptAttention takes them so)."""
        b = self.batch
        call = _Call(_device(b), stream)
        new = (b.n_kv_heads, self.total, 128)
        if self._out is None and (K_out is None or V_out is None):
            self._out = [torch.empty(*new, dtype=torch.bfloat16, device=_device(b)) for _ in range(2)]
        K_out = self._out[0] if K_out is None else K_out
        V_out = self._out[1] if V_out is None else V_out
        kv = cache.struct(call, b)
        call.run("tactic_quant_read", ctypes.byref(kv), ctypes.byref(self._shape), ctypes.byref(self._rows),
                 call.tensor(K_out, "K_out", torch.bfloat16, new), call.tensor(V_out, "V_out", torch.bfloat16, new))
        return K_out, V_out


class BlockSelector:
    """The blocks of every KV head with the best bounds for a token (tactic_block_select): `budget` of them,
    the `first` first and `last` last ones of each sequence always among them."""

    def __init__(self, batch: RaggedBatch, block: int, budget: int, first: int = 1, last: int = 2):
        self.batch, self.block = batch, int(block)
        if self.block not in BLOCKS:
            raise ValueError("block must be 16, 32, 64 or 128")
        if int(budget) < 1 or int(first) < 0 or int(last) < 0 or int(first) + int(last) > int(budget):
            raise ValueError("budget must be >= 1 and at least first + last")
        self.budget = int(budget)
        self._params = C.BlockParams(self.budget, int(first), int(last))
        self._shape = batch.struct()
        dev = _device(batch)
        name = "tactic_block_select_workspace_size"
        self.workspace = _workspace(getattr(C.lib(), name)(ctypes.byref(self._shape), self.block), name, dev)
        self.blocks = torch.empty(batch.batch, batch.n_kv_heads, self.budget, dtype=torch.int32, device=dev)
        self.counts = torch.empty(batch.batch, batch.n_kv_heads, dtype=torch.int32, device=dev)

    def __call__(self, q: torch.Tensor, cache: QuantizedCache, stream=None):
        """q bf16 [B][Hq][128] -> (blocks int32 [B][Hkv][budget], ascending and then -1; counts int32 [B][Hkv])."""
        b = self.batch
        if cache.block != self.block:
            raise ValueError(f"the cache has bounds of blocks of {cache.block} rows, expected {self.block}")
        call = _Call(_device(b), stream)
        kv = cache.struct(call, b, rows=False)
        call.run("tactic_block_select", call.tensor(q, "q", torch.bfloat16, (b.batch, b.n_q_heads, 128)), ctypes.byref(kv),
                 ctypes.byref(self._shape), ctypes.byref(self._params), self.blocks.data_ptr(), self.counts.data_ptr(),
                 self.workspace.data_ptr(), self.workspace.numel())
        return self.blocks, self.counts


class QuantizedDecoder:
    """One token per sequence over a quantised cache (tactic_quant_decode), all of its rows or those of
    chosen blocks."""

    def __init__(self, batch: RaggedBatch):
        self.batch = batch
        self._shape = batch.struct()
        dev = _device(batch)
        name = "tactic_dense_decode_workspace_size"
        self.workspace = _workspace(getattr(C.lib(), name)(ctypes.byref(self._shape)), name, dev)
        self.out = torch.empty(batch.batch, batch.n_q_heads, 128, dtype=torch.float32, device=dev)
        self.lse = torch.empty(batch.batch, batch.n_q_heads, dtype=torch.float32, device=dev)

    def __call__(self, q: torch.Tensor, cache: QuantizedCache, mod: Optional[ScoreMod] = None,
                 blocks: Optional[torch.Tensor] = None, counts: Optional[torch.Tensor] = None, stream=None,
                 out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None):
        """q bf16 [B][Hq][128] -> (out fp32 [B][Hq][128], lse fp32 [B][Hq]).  mod: a cap and slopes.  blocks int32
        [B][Hkv][budget] and counts int32 [B][Hkv], as BlockSelector gives them for the same lengths."""
        b = self.batch
        call = _Call(_device(b), stream)
        t = call.tensor
        out = self.out if out is None else out
        lse = self.lse if lse is None else lse
        if (blocks is None) != (counts is None):
            raise ValueError("blocks and counts go together")
        budget = 0
        if blocks is not None:
            if cache.block == 0:
                raise ValueError("blocks of a cache without a block size")
            if blocks.dim() != 3:
                raise ValueError(f"blocks must be [{b.batch}][{b.n_kv_heads}][budget], got {list(blocks.shape)}")
            budget = int(blocks.shape[2])
        kv = cache.struct(call, b)
        m = None if mod is None else ctypes.byref(mod.struct(call, b))
        call.run("tactic_quant_decode", t(q, "q", torch.bfloat16, (b.batch, b.n_q_heads, 128)), ctypes.byref(kv),
                 ctypes.byref(self._shape), m,
                 t(blocks, "blocks", torch.int32, (b.batch, b.n_kv_heads, budget), True),
                 t(counts, "counts", torch.int32, (b.batch, b.n_kv_heads), True), budget,
                 t(out, "out", torch.float32, (b.batch, b.n_q_heads, 128)),
                 t(lse, "lse", torch.float32, (b.batch, b.n_q_heads)), self.workspace.data_ptr(), self.workspace.numel())
        return out, lse
