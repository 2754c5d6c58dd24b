"""Matrices in MXFP4 (include/llm42_mx4.h): a buffer and its sizes around the binding's calls.  No arithmetic happens here."""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as B


class Mx4Matrix:
    """A rows x cols matrix held in 4.25 bits a value; blocks of 32 along the columns."""

    def __init__(self, data: torch.Tensor, rows: int, cols: int):
        self.data, self.rows, self.cols = data, rows, cols

    @classmethod
    def quantize(cls, src: torch.Tensor, data: Optional[torch.Tensor] = None) -> "Mx4Matrix":
        """One llm42_mx4_quantize call; src [rows, cols], bfloat16 or float32.  `data`: a uint8 tensor to hold it."""
        rows, cols = src.shape
        if data is None:
            data = torch.empty(B.llm42_mx4_bytes(rows, cols), dtype=torch.uint8, device=src.device)
        B.llm42_mx4_quantize(src, data)
        return cls(data, rows, cols)

    def values(self, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """One llm42_mx4_dequantize call: what the matrix stands for."""
        if out is None:
            out = torch.empty((self.rows, self.cols), dtype=dtype, device=self.data.device)
        if tuple(out.shape) != (self.rows, self.cols):
            raise ValueError(f"out must be [{self.rows}, {self.cols}]")
        B.llm42_mx4_dequantize(self.data, out)
        return out

    def matmul(self, x: torch.Tensor, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None,
               workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
        """One llm42_mx4_matmul call: x [m, cols] (bfloat16) times the transpose, [m, rows] in dtype (or in out's).  The workspace is allocated
        if none is given and the call makes use of one (up to 8 rows, and 16 of up to 4096 columns, are summed in one piece)."""
        if x.dim() != 2 or x.shape[1] != self.cols:
            raise ValueError(f"x must be [rows, {self.cols}]")
        if out is None:
            out = torch.empty((x.shape[0], self.rows), dtype=dtype, device=self.data.device)
        if tuple(out.shape) != (x.shape[0], self.rows):
            raise ValueError(f"out must be [{x.shape[0]}, {self.rows}]")
        few = x.shape[0] <= (16 if self.cols <= 4096 else 8) and x.data_ptr() % 4 == 0 and x.stride(0) % 2 == 0
        if workspace is None and not few:
            workspace = torch.empty(B.llm42_mx4_matmul_workspace_bytes(x.shape[0], self.rows, self.cols), dtype=torch.uint8, device=x.device)
        B.llm42_mx4_matmul(self.data, x, out, workspace)
        return out
