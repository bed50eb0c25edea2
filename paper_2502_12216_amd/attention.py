"""Attention beside the sparse decode, over the C ABI (include/tactic.h): prompts,
capped and biased scores, shared prefixes, accumulated weights and eviction.

As in tactic.py, torch supplies device memory and the current stream of the
tensors' device; every step runs in libtactic.so and a failing call raises.
Objects hold the workspace and the outputs that their calls return, so repeated
calls allocate nothing; calls of one object must be ordered on one stream.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import numpy as np
import torch

from . import _capi as C
from .tactic import PagedCache, RaggedBatch, _check_tensor, _indptr


class _Call:
    """Checks of what a call is given, and its device and stream."""

    def __init__(self, device, stream):
        self.device, self.stream = device, stream

    def tensor(self, t, name, dtype, shape=None, optional=False):
        """The pointer of tensor t after its checks (None: null, where optional)."""
        if t is None and optional:
            return None
        if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.device == self.device and t.is_cuda and
                t.is_contiguous() and (shape is None or t.shape == shape)):
            _check_tensor(t, name, dtype, shape)  # says which
            raise ValueError(f"{name} is on {t.device}, expected {self.device}")
        # (an empty tensor has no storage: any pointer that is not null stands for it)
        return t.data_ptr() or 16

    def paged(self, cache: PagedCache, batch, name: str, sequences: int):
        # (the attributes may have been replaced since the cache was made, whose sizes bound the kernels' reads)
        pages = (cache.num_pages, batch.n_kv_heads, cache.page_size, 128)
        for part in ("K_pages", "V_pages"):
            if tuple(getattr(cache, part).shape) != pages:
                raise ValueError(f"{name}.{part} must be {list(pages)}, got {list(getattr(cache, part).shape)}")
        if tuple(cache.page_table.shape) != (sequences, cache.max_pages):
            raise ValueError(f"{name}.page_table must be {[sequences, cache.max_pages]}, got {list(cache.page_table.shape)}")
        self.tensor(cache.K_pages, f"{name}.K_pages", torch.bfloat16)
        self.tensor(cache.V_pages, f"{name}.V_pages", torch.bfloat16)
        self.tensor(cache.page_table, f"{name}.page_table", torch.int32)
        return cache.struct()

    def run(self, name: str, *args):
        s = self.stream
        if s is None:
            s = torch.cuda.current_stream(self.device)
        elif s.device != self.device:
            raise ValueError(f"the stream is on {s.device}, expected {self.device}")
        f = getattr(C.lib(), name)
        if torch.cuda.current_device() == self.device.index:
            status = f(*args, s.cuda_stream)
        else:
            with torch.cuda.device(self.device):
                status = f(*args, s.cuda_stream)
        if status != C.TACTIC_OK:
            C.check(status, name)


def _device(batch: RaggedBatch):
    return batch.kv_indptr.device


def _workspace(nbytes: int, name: str, device, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    if nbytes == 0:
        C.check(1, name)
    # (a view that repeats or skips bytes is not as much memory as it has elements)
    if (workspace is not None and workspace.dtype == torch.uint8 and workspace.device == device and
            workspace.numel() >= nbytes and workspace.is_contiguous() and workspace.data_ptr() % 16 == 0):
        return workspace
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


class ScoreMod:
    """How scores are formed (see tactic_score_mod): cap in [2^-120, 2^120] caps them by cap tanh(s / cap), 0 is none;
    slopes fp32 [Hq] subtract slope |distance|; documents int32 [total] let a query see its own
    document only; prefix_len int32 [B] (prompts) lets every query see so many first tokens."""

    def __init__(self, cap: float = 0.0, slopes: Optional[torch.Tensor] = None,
                 documents: Optional[torch.Tensor] = None, prefix_len: Optional[torch.Tensor] = None):
        self.cap = float(cap)
        if self.cap != 0.0 and not 2.0 ** -120 <= self.cap <= 2.0 ** 120:
            raise ValueError("cap must be 0 or in [2^-120, 2^120]")
        self.slopes, self.documents, self.prefix_len = slopes, documents, prefix_len

    def struct(self, call: _Call, batch: RaggedBatch) -> C.ScoreMod:
        return C.ScoreMod(self.cap, call.tensor(self.slopes, "slopes", torch.float32, (batch.n_q_heads,), True),
                          call.tensor(self.documents, "documents", torch.int32, (batch.total,), True),
                          call.tensor(self.prefix_len, "prefix_len", torch.int32, (batch.batch,), True))


def _mod(mod: Optional[ScoreMod], call: _Call, batch: RaggedBatch) -> C.ScoreMod:
    return (mod if mod is not None else ScoreMod()).struct(call, batch)


def _check_kv(call, batch, K, V):
    shape = (batch.n_kv_heads, batch.total, 128)
    return call.tensor(K, "K", torch.bfloat16, shape), call.tensor(V, "V", torch.bfloat16, shape)


class PromptAttention:
    """Attention of each sequence's last q_lens[b] tokens over its cache (tactic_prompt_attention):
    a prompt (q_lens = the lengths) or a chunk of one."""

    def __init__(self, batch: RaggedBatch, q_lens: Sequence[int], workspace: Optional[torch.Tensor] = None):
        """workspace: a uint8 device tensor to use if it is large enough (for
        instance that of the chunk before), contiguous and 16-byte aligned, else a
        new one is allocated."""
        self.batch, self.q_lens = batch, [int(x) for x in q_lens]
        if len(self.q_lens) != batch.batch:
            raise ValueError("q_lens must name every sequence")
        if any(m < 0 for m in self.q_lens):
            raise ValueError("q_lens must be >= 0")
        dev = _device(batch)
        self.q_indptr_host = _indptr(self.q_lens)
        self.q_indptr = torch.as_tensor(self.q_indptr_host, device=dev)
        self.total = int(self.q_indptr_host[-1])
        self._shape = batch.struct()
        self._queries = C.QueryShape(self.total, max(self.q_lens), self.q_indptr.data_ptr())
        name = "tactic_prompt_attention_workspace_size"
        self.workspace = _workspace(getattr(C.lib(), name)(ctypes.byref(self._shape), ctypes.byref(self._queries)),
                                    name, dev, workspace)
        self.out = torch.empty(self.total, batch.n_q_heads, 128, dtype=torch.bfloat16, device=dev)
        self.lse = torch.empty(batch.n_q_heads, self.total, dtype=torch.float32, device=dev)

    def _outputs(self, call, q, out, lse):
        b = self.batch
        out = self.out if out is None else out
        lse = self.lse if lse is None else lse
        return (call.tensor(q, "q", torch.bfloat16, (self.total, b.n_q_heads, 128)), out, lse,
                call.tensor(out, "out", torch.bfloat16, (self.total, b.n_q_heads, 128)),
                call.tensor(lse, "lse", torch.float32, (b.n_q_heads, self.total)))

    def __call__(self, q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, mod: Optional[ScoreMod] = None, stream=None,
                 out=None, lse=None):
        """q bf16 [total queries][Hq][128] -> (out bf16, the same shape; lse fp32 [Hq][total queries])."""
        call = _Call(_device(self.batch), stream)
        qp, out, lse, op, lp = self._outputs(call, q, out, lse)
        kp, vp = _check_kv(call, self.batch, K, V)
        m = _mod(mod, call, self.batch)
        call.run("tactic_prompt_attention", qp, kp, vp, ctypes.byref(self._shape), ctypes.byref(self._queries),
                 ctypes.byref(m), op, lp, self.workspace.data_ptr(), self.workspace.numel())
        return out, lse

    def paged(self, q: torch.Tensor, cache: PagedCache, mod: Optional[ScoreMod] = None, stream=None, out=None, lse=None):
        """The same over a paged cache (tactic_prompt_attention_paged)."""
        call = _Call(_device(self.batch), stream)
        qp, out, lse, op, lp = self._outputs(call, q, out, lse)
        kv = call.paged(cache, self.batch, "cache", self.batch.batch)
        m = _mod(mod, call, self.batch)
        call.run("tactic_prompt_attention_paged", qp, ctypes.byref(kv), ctypes.byref(self._shape),
                 ctypes.byref(self._queries), ctypes.byref(m), op, lp, self.workspace.data_ptr(), self.workspace.numel())
        return out, lse

    def add_weights(self, q: torch.Tensor, K: torch.Tensor, lse: torch.Tensor, weights: torch.Tensor,
                    mod: Optional[ScoreMod] = None, window: int = 0, stream=None) -> torch.Tensor:
        """Adds the attention weights that the last `window` queries of every sequence (0: all) give to
        each cached row, summed over a group's heads, to weights fp32 [Hkv][total] (tactic_prompt_weights);
        lse from the call with the same arguments.  Returns weights."""
        b = self.batch
        call = _Call(_device(b), stream)
        m = _mod(mod, call, b)
        call.run("tactic_prompt_weights", call.tensor(q, "q", torch.bfloat16, (self.total, b.n_q_heads, 128)),
                 call.tensor(K, "K", torch.bfloat16, (b.n_kv_heads, b.total, 128)), ctypes.byref(self._shape),
                 ctypes.byref(self._queries), ctypes.byref(m),
                 call.tensor(lse, "lse", torch.float32, (b.n_q_heads, self.total)), int(window),
                 call.tensor(weights, "weights", torch.float32, (b.n_kv_heads, b.total)),
                 self.workspace.data_ptr(), self.workspace.numel())
        return weights


class ScoredDecoder:
    """Dense decode with capped and biased scores, documents, and caches of any
    positions (tactic_scored_decode); optionally sums the attention weights."""

    def __init__(self, batch: RaggedBatch):
        self.batch = batch
        self._shape = batch.struct()
        dev = _device(batch)
        self._ws = {}
        self._workspace(False)
        self.out = torch.empty(batch.batch, batch.n_q_heads, 128, dtype=torch.float32, device=dev)
        self.lse = torch.empty(batch.batch, batch.n_q_heads, dtype=torch.float32, device=dev)

    def _workspace(self, weights: bool) -> torch.Tensor:
        if weights not in self._ws:  # (the first call with weights sizes a second one)
            name = "tactic_scored_decode_workspace_size"
            self._ws[weights] = _workspace(getattr(C.lib(), name)(ctypes.byref(self._shape), int(weights)), name,
                                           _device(self.batch))
        return self._ws[weights]

    def _run(self, name, kv, q, mod, stream, out, lse, positions, q_pos, q_documents, weights, call):
        b = self.batch
        out = self.out if out is None else out
        lse = self.lse if lse is None else lse
        t = call.tensor
        rows = C.TokenRows(t(positions, "positions", torch.int32, (b.n_kv_heads, b.total), True),
                           t(q_pos, "q_pos", torch.int32, (b.batch,), True),
                           t(q_documents, "q_documents", torch.int32, (b.batch,), True))
        m = _mod(mod, call, b)
        qp = t(q, "q", torch.bfloat16, (b.batch, b.n_q_heads, 128))
        op = t(out, "out", torch.float32, (b.batch, b.n_q_heads, 128))
        lp = t(lse, "lse", torch.float32, (b.batch, b.n_q_heads))
        wp = t(weights, "weights", torch.float32, (b.n_kv_heads, b.total), True)
        ws = self._workspace(weights is not None)
        call.run(name, qp, *kv, ctypes.byref(self._shape), ctypes.byref(m), ctypes.byref(rows), op, lp, wp,
                 ws.data_ptr(), ws.numel())
        return out, lse

    def __call__(self, q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, mod: Optional[ScoreMod] = None,
                 positions: Optional[torch.Tensor] = None, q_pos: Optional[torch.Tensor] = None,
                 q_documents: Optional[torch.Tensor] = None, weights: Optional[torch.Tensor] = None, stream=None,
                 out=None, lse=None):
        """q bf16 [B][Hq][128] -> (out fp32 [B][Hq][128], lse fp32 [B][Hq]).  positions int32 [Hkv][total]
        (default: the row) and q_pos int32 [B] (default: the last row) for the bias; q_documents int32 [B]
        with mod.documents; weights fp32 [Hkv][total] takes this step's attention weights on top."""
        call = _Call(_device(self.batch), stream)
        return self._run("tactic_scored_decode", _check_kv(call, self.batch, K, V), q, mod, stream, out, lse, positions,
                         q_pos, q_documents, weights, call)

    def paged(self, q: torch.Tensor, cache: PagedCache, mod: Optional[ScoreMod] = None,
              positions: Optional[torch.Tensor] = None, q_pos: Optional[torch.Tensor] = None,
              q_documents: Optional[torch.Tensor] = None, weights: Optional[torch.Tensor] = None, stream=None,
              out=None, lse=None):
        """The same over a paged cache (tactic_scored_decode_paged); per-row arrays stay [..][total]."""
        call = _Call(_device(self.batch), stream)
        kv = call.paged(cache, self.batch, "cache", self.batch.batch)
        return self._run("tactic_scored_decode_paged", (ctypes.byref(kv),), q, mod, stream, out, lse, positions, q_pos,
                         q_documents, weights, call)


class SharedPrefixDecoder:
    """Decode of a batch whose sequences share long prefixes (tactic_shared_decode):
    sequence b attends prefix prefix_of[b] (negative: none), then its own tokens."""

    def __init__(self, batch: RaggedBatch, prefix_lens: Sequence[int], prefix_of: Sequence[int]):
        self.batch = batch
        self.prefix_lens, self.prefix_of = [int(x) for x in prefix_lens], [int(x) for x in prefix_of]
        if len(self.prefix_of) != batch.batch:
            raise ValueError("prefix_of must name every sequence")
        if not self.prefix_lens or any(n < 0 for n in self.prefix_lens):
            raise ValueError("prefix_lens needs a prefix, none shorter than 0")
        if any(i >= len(self.prefix_lens) for i in self.prefix_of):
            raise ValueError("prefix_of names a prefix that is not there")
        dev = _device(batch)
        members = [[b for b, i in enumerate(self.prefix_of) if i == p] for p in range(len(self.prefix_lens))]
        self.prefix_indptr = torch.as_tensor(_indptr(self.prefix_lens), device=dev)
        self.total = int(sum(self.prefix_lens))

        def ints(x):
            return torch.as_tensor(np.asarray(x, dtype=np.int32), device=dev)

        self._of, self._members = ints(self.prefix_of), ints([b for m in members for b in m] or [0])
        self._member_indptr = ints(_indptr([len(m) for m in members]))
        self._shape = batch.struct()
        self._prefixes = C.Prefixes(len(self.prefix_lens), max(len(m) for m in members), self.total,
                                    max(self.prefix_lens), self.prefix_indptr.data_ptr(), self._of.data_ptr(),
                                    self._members.data_ptr(), self._member_indptr.data_ptr(),
                                    sum(len(m) for m in members))
        name = "tactic_shared_decode_workspace_size"
        self.workspace = _workspace(getattr(C.lib(), name)(ctypes.byref(self._shape), ctypes.byref(self._prefixes)),
                                    name, dev)
        self.out = torch.empty(batch.batch, batch.n_q_heads, 128, dtype=torch.float32, device=dev)
        self.lse = torch.empty(batch.batch, batch.n_q_heads, dtype=torch.float32, device=dev)

    def _run(self, name, kv, q, mod, out, lse, call):
        b = self.batch
        out = self.out if out is None else out
        lse = self.lse if lse is None else lse
        m = _mod(mod, call, b)
        call.run(name, call.tensor(q, "q", torch.bfloat16, (b.batch, b.n_q_heads, 128)), *kv, ctypes.byref(self._shape),
                 ctypes.byref(self._prefixes), ctypes.byref(m),
                 call.tensor(out, "out", torch.float32, (b.batch, b.n_q_heads, 128)),
                 call.tensor(lse, "lse", torch.float32, (b.batch, b.n_q_heads)),
                 self.workspace.data_ptr(), self.workspace.numel())
        return out, lse

    def __call__(self, q: torch.Tensor, K_prefix: torch.Tensor, V_prefix: torch.Tensor, K: torch.Tensor,
                 V: torch.Tensor, mod: Optional[ScoreMod] = None, stream=None, out=None, lse=None):
        """q bf16 [B][Hq][128], K_prefix, V_prefix bf16 [Hkv][total prefix tokens][128], K, V the sequences' own
        tokens -> (out fp32 [B][Hq][128], lse fp32 [B][Hq]).  mod: a cap and slopes; positions count the prefix."""
        call = _Call(_device(self.batch), stream)
        shape = (self.batch.n_kv_heads, self.total, 128)
        kv = (call.tensor(K_prefix, "K_prefix", torch.bfloat16, shape), call.tensor(V_prefix, "V_prefix", torch.bfloat16, shape),
              *_check_kv(call, self.batch, K, V))
        return self._run("tactic_shared_decode", kv, q, mod, out, lse, call)

    def paged(self, q: torch.Tensor, prefix_cache: PagedCache, cache: PagedCache, mod: Optional[ScoreMod] = None,
              stream=None, out=None, lse=None):
        """The same over paged caches (tactic_shared_decode_paged): prefix_cache's page table has a row per
        prefix; both may use the same page arrays."""
        call = _Call(_device(self.batch), stream)
        kv = (call.paged(prefix_cache, self.batch, "prefix_cache", len(self.prefix_lens)),
              call.paged(cache, self.batch, "cache", self.batch.batch))
        return self._run("tactic_shared_decode_paged", tuple(ctypes.byref(x) for x in kv), q, mod, out, lse, call)


class CacheEvictor:
    """Keeps the recent rows and those of the largest accumulated attention weights,
    in another cache (tactic_evict)."""

    def __init__(self, batch: RaggedBatch, dest: RaggedBatch, recent: int):
        """dest: the other cache's batch, with capacities; its seq_len is set by each call on the device
        (dest.seq_lens, on the host, is the caller's to keep)."""
        if dest.batch != batch.batch or dest.n_kv_heads != batch.n_kv_heads:
            raise ValueError("dest must have the same sequences and KV heads")
        if dest.seq_len is None:
            raise ValueError("dest needs capacities")
        if dest.seq_len is batch.seq_len:
            raise ValueError("dest must be another batch: its lengths are set while the batch's are read")
        self.batch, self.dest, self.recent = batch, dest, int(recent)
        self._shape = batch.struct()
        name = "tactic_evict_workspace_size"
        self.workspace = _workspace(getattr(C.lib(), name)(ctypes.byref(self._shape), dest.total), name, _device(batch))

    def __call__(self, K: torch.Tensor, V: torch.Tensor, weights: torch.Tensor, keep: torch.Tensor, K_out: torch.Tensor,
                 V_out: torch.Tensor, weights_out: torch.Tensor, positions_out: torch.Tensor,
                 positions: Optional[torch.Tensor] = None, newest: Optional[torch.Tensor] = None, stream=None) -> None:
        """keep int32 [B]: rows that each sequence keeps (at most what it has and its capacity); weights fp32 and
        positions int32 (default: the row) [Hkv][total]; newest int32 [B] the last position (default: the last
        row).  K_out, V_out, weights_out, positions_out: [Hkv][dest.total]..."""
        b, d = self.batch, self.dest
        call = _Call(_device(b), stream)
        t = call.tensor
        kp, vp = _check_kv(call, b, K, V)
        rows, outs = (b.n_kv_heads, b.total), (b.n_kv_heads, d.total)
        call.run("tactic_evict", kp, vp, ctypes.byref(self._shape), t(weights, "weights", torch.float32, rows),
                 t(positions, "positions", torch.int32, rows, True), t(keep, "keep", torch.int32, (b.batch,)),
                 t(newest, "newest", torch.int32, (b.batch,), True), self.recent,
                 t(d.kv_indptr, "dest.kv_indptr", torch.int64), d.total, d.max_len,
                 t(K_out, "K_out", torch.bfloat16, outs + (128,)), t(V_out, "V_out", torch.bfloat16, outs + (128,)),
                 t(weights_out, "weights_out", torch.float32, outs), t(positions_out, "positions_out", torch.int32, outs),
                 t(d.seq_len, "dest.seq_len", torch.int64), self.workspace.data_ptr(), self.workspace.numel())


class TokenInserter:
    """A new token for every sequence of a cache: behind the last row while its span has room,
    else in place of the row that eviction would drop first (tactic_insert_token)."""

    def __init__(self, batch: RaggedBatch, recent: int):
        if batch.seq_len is None:
            raise ValueError("batch needs capacities")
        self.batch, self.recent = batch, int(recent)
        self._shape = batch.struct()
        self.rows = torch.empty(batch.batch, batch.n_kv_heads, dtype=torch.int32, device=_device(batch))

    def __call__(self, k: torch.Tensor, v: torch.Tensor, K: torch.Tensor, V: torch.Tensor, weights: torch.Tensor,
                 positions: torch.Tensor, newest: torch.Tensor, stream=None) -> torch.Tensor:
        """k, v bf16 [B][Hkv][128] at positions newest int32 [B]; K, V, weights and positions are changed in
        place and batch.seq_len grows up to the capacities (batch.seq_lens, on the host, is the caller's to
        keep).  Returns the rows int32 [B][Hkv] that the tokens went to."""
        b = self.batch
        call = _Call(_device(b), stream)
        t = call.tensor
        kp, vp = _check_kv(call, b, K, V)
        rows = (b.n_kv_heads, b.total)
        one = (b.batch, b.n_kv_heads, 128)
        call.run("tactic_insert_token", t(k, "k", torch.bfloat16, one), t(v, "v", torch.bfloat16, one),
                 t(newest, "newest", torch.int32, (b.batch,)), self.recent, ctypes.byref(self._shape),
                 b.seq_len.data_ptr(), kp, vp, t(weights, "weights", torch.float32, rows),
                 t(positions, "positions", torch.int32, rows), self.rows.data_ptr())
        return self.rows
