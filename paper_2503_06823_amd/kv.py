"""The paged 4-bit key/value cache of a model's attention layers, for a batch of requests: buffers and call order.  All
arithmetic, the tables included, is in libemoe; nothing here waits for the GPU.

One step of a batch, all its tensors on one stream:

    kv.plan(new_len, T)            # pages, slots and positions of the step's T tokens (new_len[r] of request r, in row order)
    for every attention layer:
        kv.append(layer, k, v)     # the step's keys and values, after the positions have been applied to them
        kv.attend(layer, q, out, max_new)
    kv.release(ended)              # pages that nobody will read again

A step leaves every buffer where it was: one that was captured in a graph replays as the next one.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import List, Optional

import torch

from . import binding as B

MOST_WORKSPACE = 64 << 20  # no call needs more
ELEMENTS = {B.EMOE_F32: torch.float32, B.EMOE_BF16: torch.bfloat16}


def _described(t) -> str:
    return f"{t.dtype} {list(t.shape)} with strides {list(t.stride())} on {t.device}" if isinstance(t, torch.Tensor) else repr(t)


@dataclass
class KvCache:
    """Caches of the attention layers, the tables that they share, and the ring of free pages.  `window` and `sinks`: of the
    layers' sliding window (0: none); a page leaves once it is out of every layer's sight, so all layers have the same."""
    desc: B.EmoeKvDesc
    dtype: str
    window: int
    sinks: int
    caches: List[torch.Tensor]      # one a layer, uint8 [pages, kv_heads, bytes of a page]
    block_table: torch.Tensor       # int32 [rows, table_width]
    free_pages: torch.Tensor        # int32 [pages], a ring
    counters: List[torch.Tensor]    # its int64 {head, tail}, twice: every call reads one and writes the other
    length: List[torch.Tensor]      # int32 [rows], twice: tokens held between steps; in the last step, its own included (0: refused)
    cu_new: torch.Tensor
    slot: torch.Tensor
    position: torch.Tensor
    refused: torch.Tensor           # rows that got no pages in the last plan(): their outputs are zeros, their length is 0
    ws: torch.Tensor
    T: int = 0

    @staticmethod
    def allocate(layers: int, rows: int, max_tokens: int, pages: int, page_size: int, kv_heads: int, head_dim: int, most_new: int,
                 dtype: str = "bf16", window: int = 0, sinks: int = 0, device="cuda:0") -> "KvCache":
        """`max_tokens`: of a request; `most_new`: tokens of a step, all requests together."""
        desc = B.make_kv_desc(pages, page_size, kv_heads, head_dim, rows, -(-max_tokens // page_size))
        n = B.emoe_kv_cache_bytes(desc)
        i32 = dict(dtype=torch.int32, device=device)
        zeros = lambda k: torch.zeros(max(k, 1), **i32)
        return KvCache(
            desc=desc, dtype=dtype, window=window, sinks=sinks,
            caches=[torch.empty((pages, kv_heads, n // (pages * kv_heads)), dtype=torch.uint8, device=device) for _ in range(layers)],
            block_table=torch.full((rows, desc.table_width), -1, **i32), free_pages=torch.arange(pages, **i32),
            counters=[torch.tensor([0, pages], dtype=torch.int64, device=device), torch.zeros(2, dtype=torch.int64, device=device)],
            length=[zeros(rows), zeros(rows)], cu_new=zeros(rows + 1), slot=zeros(most_new), position=zeros(most_new), refused=zeros(1),
            ws=torch.empty(MOST_WORKSPACE, dtype=torch.uint8, device=device))

    def __post_init__(self):
        self._element, self._device = ELEMENTS[B.DTYPES.get(self.dtype, self.dtype)], self.slot.device
        self._kv_heads, self._dim = self.desc.kv_heads, self.desc.head_dim

    # The library is handed addresses and strides: what these would not say is checked here, before anything is enqueued.  (A microsecond a tensor:
    # a tensor's shape and strides are asked for once.)
    def _check_per_request(self, name: str, t: torch.Tensor) -> None:
        if not (isinstance(t, torch.Tensor) and t.dtype is torch.int32 and t.shape == (self.desc.rows,) and t.device == self._device and t.is_contiguous()):
            raise ValueError(f"{name}: int32 [{self.desc.rows}] on {self._device}, dense, is wanted, not {_described(t)}")

    def _row_stride(self, name: str, t: torch.Tensor, heads: int) -> int:
        """Elements from one token's row to the next, of a tensor that has rows for the step's tokens."""
        row = heads * self._dim
        if isinstance(t, torch.Tensor) and t.dtype is self._element and t.device == self._device and t.dim() == 3:
            (tokens, its_heads, dim), (by_token, by_head, by_element) = t.shape, t.stride()
            if tokens >= self.T and its_heads == heads and dim == self._dim and by_element == 1 and (by_head == dim or heads == 1):
                if self.T <= 1:
                    return row  # a single row's own stride says nothing
                if by_token >= row:
                    return by_token
        raise ValueError(f"{name}: {self._element} [{self.T} or more, {heads}, {self._dim}] on {self._device} with dense rows is wanted, not {_described(t)}")

    def plan(self, new_len: torch.Tensor, T: int, stream=None) -> None:
        """`new_len`: int32 [rows] on the device; `T`: their sum, at most the most_new of allocate()."""
        if not 0 <= T <= self.slot.numel():
            raise ValueError(f"{T} tokens in a step for buffers of {self.slot.numel()}")
        self._check_per_request("new_len", new_len)
        held, after = self.length
        B.emoe_kv_plan(self.desc, T, held, new_len, self.block_table, self.free_pages, self.counters[0], self.cu_new, self.slot,
                       self.position, after, self.counters[1], self.refused, stream)
        self.counters.reverse()
        self.T = T

    def append(self, layer: int, k: torch.Tensor, v: torch.Tensor, stream=None) -> None:
        """`k`, `v`: [T, kv_heads, head_dim], each a slice of a wider row if need be."""
        k_stride, v_stride = self._row_stride("k", k, self._kv_heads), self._row_stride("v", v, self._kv_heads)
        B.emoe_kv_append(self.desc, self.T, self.dtype, k, v, self.slot, self.caches[layer], k_stride, v_stride, stream)

    def attend(self, layer: int, q: torch.Tensor, out: torch.Tensor, max_new: int, scale: Optional[float] = None, stream=None) -> torch.Tensor:
        """`q`, `out`: [T, q_heads, head_dim], each a slice of a wider row if need be; no request has more than `max_new` new tokens (of one that
        does, the first are answered)."""
        heads = q.shape[1] if isinstance(q, torch.Tensor) and q.dim() == 3 else 0
        if heads == 0 or heads % self._kv_heads != 0:
            raise ValueError(f"q: a multiple of {self._kv_heads} heads is wanted, not {_described(q)}")
        q_stride, out_stride = self._row_stride("q", q, heads), self._row_stride("out", out, heads)
        at = B.make_attention_desc(self.T, heads, self._dim, self.dtype, min(max_new, self.T), self.window, self.sinks, scale, q_stride, out_stride)
        B.emoe_kv_attention(self.desc, at, q, self.caches[layer], self.block_table, self.length[1], self.cu_new, out, self.ws, self.ws.numel(),
                            stream)
        return out

    def release(self, ended: Optional[torch.Tensor] = None, stream=None) -> None:
        """Ends the step: rows with `ended` != 0 (int32 [rows] on the device, None: nobody) give all their pages back and start
        anew, rows that were refused keep what they held."""
        if ended is not None:
            self._check_per_request("ended", ended)
        held, after = self.length
        B.emoe_kv_release(self.desc, held, after, ended, self.window, self.sinks, self.block_table, self.free_pages, self.counters[0],
                          self.counters[1], stream)
        B.emoe_kv_advance(self.desc, after, ended, held, stream)
        self.counters.reverse()
