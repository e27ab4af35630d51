"""Matrices in 8 bits: e4m3 codes under a power of two per 128 x 128 block, half the bytes of bf16, and the products of bf16 rows with them.  All
arithmetic is in libemoe; nothing here waits for the GPU.

    m = PackedMatrices.pack(w)                  # [N, K], or [count, N, K]: one a group
    ws = m.workspace(most_rows)                 # one for all products of a stream
    m.matmul(x, out, ws)                        # out[r] = x[r] W^T
    m.matmul(x, out, ws, group_offsets)         # rows group_offsets[g] .. group_offsets[g + 1] - 1 with the g-th matrix

An MoE layer whose descriptor has the type "f8" takes its experts' matrices so: PackedMatrices.data where the slots' weights go.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Optional

import torch

from . import binding as B
from .kv import ELEMENTS, _described


@dataclass
class PackedMatrices:
    N: int
    K: int
    data: torch.Tensor  # uint8 [count, bytes of a matrix]

    @staticmethod
    def allocate(count: int, N: int, K: int, device="cuda:0") -> "PackedMatrices":
        """Room for `count` matrices, not yet written."""
        return PackedMatrices(N, K, torch.empty((count, B.emoe_matrix_bytes(N, K)), dtype=torch.uint8, device=device))

    @staticmethod
    def pack(w: torch.Tensor, stream=None) -> "PackedMatrices":
        """`w`: [N, K] or [count, N, K], fp32 or bf16, in a GPU's memory (as every tensor here: the calls refuse the host's)."""
        if not (isinstance(w, torch.Tensor) and w.dim() in (2, 3)):
            raise ValueError(f"w: [N, K] or [count, N, K] is wanted, not {_described(w)}")
        m = PackedMatrices.allocate(w.shape[0] if w.dim() == 3 else 1, w.shape[-2], w.shape[-1], w.device)
        m.write(w, stream)
        return m

    def __post_init__(self):
        if not (isinstance(self.data, torch.Tensor) and self.data.dtype is torch.uint8 and self.data.dim() == 2 and self.data.is_contiguous()
                and self.data.shape[0] > 0 and self.data.shape[1] == B.emoe_matrix_bytes(self.N, self.K)):
            raise ValueError(f"data: uint8 [count, {B.emoe_matrix_bytes(self.N, self.K)}], dense, is wanted, not {_described(self.data)}")
        self.count, self._device = self.data.shape[0], self.data.device

    # The library is handed addresses and strides: what these would not say is checked here, before anything is enqueued.
    def _check_device(self) -> None:
        if self._device.type == "cuda" and self._device.index != torch.cuda.current_device():
            raise ValueError(f"matrices on {self._device} while cuda:{torch.cuda.current_device()} is the current device")

    def _matrices(self, name: str, w: torch.Tensor):
        """(type, elements from row to row) of plain matrices."""
        if isinstance(w, torch.Tensor) and w.device == self._device and w.dtype in ELEMENTS.values() and w.dim() in (2, 3):
            whole = w if w.dim() == 3 else w[None]
            by_matrix, by_row, by_element = whole.stride()
            if tuple(whole.shape) == (self.count, self.N, self.K) and by_element == 1 and by_row >= self.K \
                    and (self.count == 1 or by_matrix == self.N * by_row):
                return B.EMOE_F32 if w.dtype is torch.float32 else B.EMOE_BF16, by_row
        raise ValueError(f"{name}: fp32 or bf16 [{self.count}, {self.N}, {self.K}] on {self._device}, dense rows at one distance, is wanted, not {_described(w)}")

    def write(self, w: torch.Tensor, stream=None) -> None:
        """Packs [count, N, K] (or [N, K] of one) in place of what was held."""
        dtype, stride = self._matrices("w", w)
        self._check_device()
        B.emoe_matrix_pack(self.count, self.N, self.K, dtype, w, self.data, stride, stream)

    def read(self, w: torch.Tensor, stream=None) -> torch.Tensor:
        """The numbers that the matrices hold, into fp32 or bf16 [count, N, K] (or [N, K] of one): exact in both."""
        dtype, stride = self._matrices("w", w)
        self._check_device()
        B.emoe_matrix_unpack(self.count, self.N, self.K, dtype, self.data, w, stride, stream)
        return w

    def _desc(self, rows: int, x_stride: int, out_stride: int) -> B.EmoeMatmulDesc:
        return B.make_matmul_desc(rows, self.N, self.K, self.count, "bf16", x_stride, out_stride)

    def workspace_bytes(self, rows: int) -> int:
        """Of products of up to `rows` rows."""
        return B.emoe_matmul_workspace_bytes(self._desc(rows, self.K, self.N))

    def workspace(self, rows: int) -> torch.Tensor:
        return torch.empty(max(self.workspace_bytes(rows), 1), dtype=torch.uint8, device=self._device)

    def _row_stride(self, name: str, t: torch.Tensor, elements: int) -> int:
        if isinstance(t, torch.Tensor) and t.dtype is torch.bfloat16 and t.device == self._device and t.dim() == 2 and t.shape[1] == elements:
            by_row, by_element = t.stride()
            if by_element == 1:
                if t.shape[0] <= 1:
                    return elements  # a single row's own stride says nothing
                if by_row >= elements:
                    return by_row
        raise ValueError(f"{name}: bf16 [rows, {elements}] on {self._device} with dense rows is wanted, not {_described(t)}")

    def matmul(self, x: torch.Tensor, out: torch.Tensor, ws: torch.Tensor, group_offsets: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """`x` [rows, K], `out` [rows, N] bf16, each a slice of wider rows if need be; `group_offsets`: int32 [count + 1] on the device, ascending
        from 0 (rows behind the last are left as they are), to be left out with one matrix only.  `ws` is not shared with a call that may run at the same time."""
        x_stride, out_stride = self._row_stride("x", x, self.K), self._row_stride("out", out, self.N)
        rows = x.shape[0]
        if out.shape[0] != rows:
            raise ValueError(f"out: {rows} rows are wanted, not {_described(out)}")
        at = group_offsets
        if at is None:
            if self.count > 1:
                raise ValueError(f"group_offsets are wanted where there are {self.count} matrices")
        elif not (isinstance(at, torch.Tensor) and at.dtype is torch.int32 and at.shape == (self.count + 1,) and at.device == self._device
                  and at.is_contiguous()):
            raise ValueError(f"group_offsets: int32 [{self.count + 1}] on {self._device}, dense, is wanted, not {_described(at)}")
        if not (isinstance(ws, torch.Tensor) and ws.dtype is torch.uint8 and ws.device == self._device and ws.is_contiguous()):
            raise ValueError(f"ws: uint8 on {self._device}, dense, is wanted, not {_described(ws)}")
        self._check_device()
        B.emoe_matmul(self._desc(rows, x_stride, out_stride), x, at, self.data, out, ws, ws.numel(), stream)
        return out
