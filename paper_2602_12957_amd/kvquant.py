"""A paged KV cache in 8 bits: the device buffers and the calls on them.

`QuantKV` owns the pages (e4m3 codes, one power-of-two scale for each block of 16 tokens and kv head), the block tables, the
lengths and the free stack; the arithmetic runs inside libhsd.so (include/hsd.h: hsd_kv_reserve, hsd_kv_quant_append,
hsd_kv_quant_read, hsd_kv_quant_attention, hsd_kv_commit_rows).  Every call enqueues on torch's current stream of the
cache's device and returns; nothing waits.  A step of a decoder on it:

    slots, pos = cache.reserve(cu_q, total_q)          # places and positions of the new rows, one for all layers
    for l in range(n_layers):
        cache.append(k, v, slots, layer=l)             # [total_q, n_kv_heads, 64], rotary positions applied
        o = cache.attend(q, cu_q, layer=l)             # [total_q, n_q_heads, 64]
    cache.commit(cu_q, total_q)                        # or commit(cu_q, total_q, accept_len) after a verification
"""
from __future__ import annotations

import math
from typing import Optional, Tuple

import torch

from . import binding as B

_TYPES = {torch.bfloat16: B.HSD_BF16, torch.float32: B.HSD_FP32}
_HD = B.HSD_HEAD_DIM
_PAGE = B.HSD_KV_BLOCK_TOKENS * _HD


def _rows3(name: str, t: torch.Tensor, rows: int, heads: int, index: int, dtype=None) -> int:
    """A [rows, heads, 64] tensor whose rows may lie apart; returns the distance of its rows in elements."""
    if not isinstance(t, torch.Tensor) or t.get_device() != index:
        raise ValueError(f"{name} must be a tensor on cuda:{index}")
    if t.dtype not in _TYPES or (dtype is not None and t.dtype != dtype):
        raise ValueError(f"{name}: bfloat16 or float32, the same for all tensors of a call; got {t.dtype}")
    if t.shape != (rows, heads, _HD):
        raise ValueError(f"{name} must be [{rows}, {heads}, {_HD}], got {tuple(t.shape)}")
    if t.is_contiguous():
        return heads * _HD
    s = t.stride()
    if s[2] != 1 or (heads > 1 and s[1] != _HD) or (rows > 1 and s[0] < heads * _HD):
        raise ValueError(f"{name}: the heads of a row must lie one after the other and rows must not overlap")
    return s[0] if rows > 1 else heads * _HD


def _ints(name: str, t: torch.Tensor, n: int, index: int) -> int:
    if not isinstance(t, torch.Tensor) or t.get_device() != index or t.dtype != torch.int32 or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor on cuda:{index}")
    if t.dim() != 1 or (n >= 0 and t.shape[0] != n):
        raise ValueError(f"{name} must be [{n if n >= 0 else 'n_seq + 1'}], got {tuple(t.shape)}")
    return t.data_ptr()


class QuantKV:
    def __init__(self, n_blocks: int, n_kv_heads: int, n_slots: int, max_blocks_per_seq: int, n_layers: int = 1,
                 device: str = "cuda:0"):
        if min(n_blocks, n_kv_heads, n_slots, max_blocks_per_seq, n_layers) < 1:
            raise ValueError("every size of the cache must be positive")
        if not torch.cuda.is_available():
            raise RuntimeError("the 8-bit cache needs a GPU (MI355X); there is no CPU fallback")
        self.dev = torch.device(device)
        if self.dev.type != "cuda":
            raise ValueError(f"the cache lives on a GPU, not on {device}")
        if self.dev.index is None:
            self.dev = torch.device("cuda", torch.cuda.current_device())
        self._index = self.dev.index
        self.n_blocks, self.n_kv_heads, self.n_slots, self.maxb, self.n_layers = n_blocks, n_kv_heads, n_slots, max_blocks_per_seq, n_layers
        shape = (n_layers, n_blocks, n_kv_heads)
        self.k_codes = torch.zeros(shape + (_PAGE,), dtype=torch.uint8, device=self.dev)
        self.v_codes = torch.zeros(shape + (_PAGE,), dtype=torch.uint8, device=self.dev)
        self.k_scale = torch.ones(shape, dtype=torch.float32, device=self.dev)
        self.v_scale = torch.ones(shape, dtype=torch.float32, device=self.dev)
        # the bookkeeping in one buffer: a snapshot is one copy
        n_state = n_blocks + 1 + n_slots + n_slots * max_blocks_per_seq + 1
        self._state = torch.zeros(n_state, dtype=torch.int32, device=self.dev)
        self._snapshot = torch.zeros_like(self._state)
        self.free_list, self.free_count, self.seq_len, table, self.status = self._state.split(
            [n_blocks, 1, n_slots, n_slots * max_blocks_per_seq, 1])
        self.block_table = table.view(n_slots, max_blocks_per_seq)
        self.cpool = B.hsd_kv_pool(None, None, n_blocks, self.free_list.data_ptr(), self.free_count.data_ptr())
        # what every call's batch has in common: calls copy it, so that two threads do not share one
        rows = B.hsd_batch()
        rows.max_blocks_per_seq, rows.n_slots = max_blocks_per_seq, n_slots
        rows.seq_len, rows.block_table, rows.status = self.seq_len.data_ptr(), self.block_table.data_ptr(), self.status.data_ptr()
        self._rows = bytes(rows)
        self._ws_bytes = {}
        self._layers = [B.hsd_kv_quant(self.k_codes[l].data_ptr(), self.v_codes[l].data_ptr(), self.k_scale[l].data_ptr(),
                                       self.v_scale[l].data_ptr(), n_blocks, n_kv_heads) for l in range(n_layers)]
        self.reset()

    @property
    def stream(self) -> int:
        return B.current_stream(self._index)

    def reset(self):
        """Every block free, every sequence empty (the pages keep their bytes)."""
        with B.on_device(self._index):
            self.seq_len.zero_()
            self.block_table.fill_(-1)
            self.status.zero_()
            B.hsd_kv_pool_init(self.stream, self.cpool)

    def snapshot(self):
        """Remembers lengths, block tables, the free stack and status; pages are not copied."""
        self._snapshot.copy_(self._state)

    def restore(self):
        """Returns the bookkeeping to the last snapshot (one copy on the current stream)."""
        self._state.copy_(self._snapshot)

    def _batch(self, cu_q, total_q, seq_slot=None, accept_len=None) -> B.hsd_batch:
        b = B.hsd_batch.from_buffer_copy(self._rows)
        b.cu_q = _ints("cu_q", cu_q, -1, self._index)
        n = cu_q.shape[0] - 1
        if n < 1 or total_q < 0 or (seq_slot is None and n > self.n_slots):
            raise ValueError(f"bad rows: n_seq={n}, total_q={total_q}, slots={self.n_slots}")
        b.n_seq, b.total_q = n, total_q
        if seq_slot is not None:
            b.seq_slot = _ints("seq_slot", seq_slot, n, self._index)
        if accept_len is not None:
            b.accept_len = _ints("accept_len", accept_len, n, self._index)
        return b

    def _layer(self, layer: int) -> B.hsd_kv_quant:
        if not 0 <= layer < self.n_layers:
            raise ValueError(f"layer {layer} of {self.n_layers}")
        return self._layers[layer]

    def reserve(self, cu_q: torch.Tensor, total_q: int, seq_slot: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """Blocks for total_q new rows, sequence s owning rows cu_q[s] .. cu_q[s + 1] - 1 behind its seq_len tokens.
        Returns (row_slot, row_pos), int32 [total_q]; row_slot is -1 where the pool or the table is too small (see status).
        Rows from cu_q[n_seq] on, as in a padded batch, have slot -1 and position 0: append leaves them out, attend their output."""
        b = self._batch(cu_q, total_q, seq_slot)
        slot = torch.empty(total_q, dtype=torch.int32, device=self.dev)
        pos = torch.empty(total_q, dtype=torch.int32, device=self.dev)
        with B.on_device(self._index):
            B.hsd_kv_reserve(self.stream, self.cpool, b, slot.data_ptr(), pos.data_ptr())
        return slot, pos

    def commit(self, cu_q: torch.Tensor, total_q: int, accept_len: Optional[torch.Tensor] = None,
               seq_slot: Optional[torch.Tensor] = None):
        """seq_len grows by all rows of a sequence, or by 1 + accept_len[s] (not at all where it is negative); blocks that
        are wholly beyond return to the pool."""
        b = self._batch(cu_q, total_q, seq_slot, accept_len)
        with B.on_device(self._index):
            B.hsd_kv_commit_rows(self.stream, self.cpool, b)

    def append(self, k: torch.Tensor, v: torch.Tensor, row_slot: torch.Tensor, layer: int = 0):
        """Keys and values [rows, n_kv_heads, 64] into the pages at row_slot (as reserve returned it)."""
        slots, n, kv = _ints("row_slot", row_slot, -1, self._index), row_slot.shape[0], self._layer(layer)
        ks, vs = _rows3("k", k, n, self.n_kv_heads, self._index), _rows3("v", v, n, self.n_kv_heads, self._index, k.dtype)
        with B.on_device(self._index):
            B.hsd_kv_quant_append(self.stream, kv, n, slots, _TYPES[k.dtype], k.data_ptr(), v.data_ptr(), ks, vs, self.status.data_ptr())

    def read(self, row_slot: torch.Tensor, dtype: torch.dtype = torch.bfloat16, layer: int = 0) -> Tuple[torch.Tensor, torch.Tensor]:
        """The values that the cache holds at the given slots: (k, v) [rows, n_kv_heads, 64], exact in both types."""
        if dtype not in _TYPES:
            raise ValueError(f"bfloat16 or float32, got {dtype}")
        slots, n, kv, w = _ints("row_slot", row_slot, -1, self._index), row_slot.shape[0], self._layer(layer), self.n_kv_heads * _HD
        k = torch.empty((n, self.n_kv_heads, _HD), dtype=dtype, device=self.dev)
        v = torch.empty((n, self.n_kv_heads, _HD), dtype=dtype, device=self.dev)
        with B.on_device(self._index):
            B.hsd_kv_quant_read(self.stream, kv, n, slots, _TYPES[dtype], k.data_ptr(), v.data_ptr(), w, w)
        return k, v

    def attend(self, q: torch.Tensor, cu_q: torch.Tensor, seq_slot: Optional[torch.Tensor] = None, layer: int = 0,
               scale: Optional[float] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Causal attention of the rows q [rows, n_q_heads, 64] over their sequences: row i of a sequence sees its seq_len
        tokens and rows 0 .. i, whose keys and values have been appended.  scale: 1 / sqrt(64) by default; out: may be q."""
        if not isinstance(q, torch.Tensor) or q.dim() != 3 or q.shape[1] < 1 or q.shape[1] % self.n_kv_heads:
            raise ValueError(f"q must be [rows, n_q_heads, 64] with a multiple of {self.n_kv_heads} heads")
        n, heads, _ = q.shape
        kv, b = self._layer(layer), self._batch(cu_q, n, seq_slot)
        qs = _rows3("q", q, n, heads, self._index)
        if out is None:
            out, os = torch.empty((n, heads, _HD), dtype=q.dtype, device=self.dev), heads * _HD
        else:
            os = _rows3("out", out, n, heads, self._index, q.dtype)
        key = (n, b.n_seq, heads)
        nb = self._ws_bytes.get(key)
        if nb is None:
            if len(self._ws_bytes) > 4096:
                self._ws_bytes.clear()
            nb = self._ws_bytes[key] = B.hsd_kv_quant_attention_bytes(kv, b, heads)
        ws = torch.empty(nb, dtype=torch.uint8, device=self.dev) if nb else None
        with B.on_device(self._index):
            B.hsd_kv_quant_attention(self.stream, kv, b, heads, _TYPES[q.dtype], 1.0 / math.sqrt(_HD) if scale is None else float(scale),
                                     q.data_ptr(), qs, out.data_ptr(), os, ws.data_ptr() if nb else None, nb)
        return out
