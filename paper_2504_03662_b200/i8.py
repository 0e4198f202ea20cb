"""Matrices in 8-bit integers with one scale a row, and their products: a scale for each token on one side, for each output channel on the other.

The functions allocate their results through PyTorch and call the library's kernels on the current stream of the tensors' device; formats and formulas
are those of include/galv.h.  Weights are packed once (`pack`) and kept; `linear` puts a layer's input into 8-bit integers in the call.  `mx.linear` with
`eight` multiplies so in its forward pass and has gradients; experts.matmul takes weights held so for many experts.  Captures in CUDA graphs, contexts and waits that have run out: as in mx.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as gb
from .mx import _bytes, _device, _kind, _on, _rows, _vector


def pitch(cols: int) -> int:
    """Bytes of a row of codes."""
    return (cols + 15) // 16 * 16


class Packed:
    """A matrix [rows][cols] in 8-bit integers: codes int8 [rows][pitch(cols)], zeros behind a row's end, and scales fp32 [rows]."""
    __slots__ = ("codes", "scales", "rows", "cols", "device")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, rows: int, cols: int):
        if rows < 0 or cols < 1:
            raise ValueError(f"no matrix of {rows} rows and {cols} columns")
        if codes.dtype != torch.int8 or codes.numel() < rows * pitch(cols) or not codes.is_contiguous() or codes.is_neg() or (rows and codes.data_ptr() % 16):
            raise ValueError(f"a [{rows}][{cols}] matrix takes {rows * pitch(cols)} contiguous codes of int8, 16-byte aligned, got {codes.dtype} {tuple(codes.shape)}")
        if scales.dtype != torch.float32 or scales.numel() < rows or not scales.is_contiguous() or scales.is_neg():
            raise ValueError(f"{rows} rows take {rows} contiguous scales of float32, got {scales.dtype} {tuple(scales.shape)}")
        if codes.device != scales.device:
            raise ValueError(f"codes on {codes.device} and scales on {scales.device}")
        self.codes, self.scales, self.rows, self.cols, self.device = codes, scales, rows, cols, codes.device

    @property
    def nbytes(self) -> int:
        return self.rows * (pitch(self.cols) + 4)


def pack(x: torch.Tensor) -> Packed:
    """Holds a matrix in 8-bit integers."""
    _kind(x.dtype, "x")
    x = _rows(x, "x")
    g = _on(x.device)
    rows, cols = x.shape
    if cols < 1:
        raise ValueError("rows of at least one column")
    p = Packed(torch.empty(rows, pitch(cols), dtype=torch.int8, device=x.device), torch.empty(rows, dtype=torch.float32, device=x.device), rows, cols)
    g.galv_i8_pack(x, p.codes, p.scales)
    return p


def unpack(p: Packed, dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """The numbers a packed matrix stands for."""
    _kind(dtype, "dtype")
    g = _on(p.device)
    x = torch.empty(p.rows, p.cols, dtype=dtype, device=p.device)
    g.galv_i8_unpack(p.codes, p.scales, x)
    return x


def _room(rows: int, cols: int) -> int:
    """Bytes of workspace in which a product puts its input into 8-bit integers: codes in rows of whole pieces of 32, then scales, each in whole pieces of 256."""
    return (rows * ((cols + 31) // 32 * 32) + 255 & ~255) + (rows * 4 + 255 & ~255)


def _beside(cols: int, b: Packed):
    if cols != b.cols or b.rows < 1:
        raise ValueError(f"a product of {cols} columns and [{b.rows}][{b.cols}] transposed")
    if cols > gb.I8_MOST:
        raise ValueError(f"products of 8-bit integers sum up to {gb.I8_MOST} columns, not {cols}")


def _bias(bias: Optional[torch.Tensor], shape, dtype: torch.dtype):
    if bias is not None and (bias.dtype != dtype or tuple(bias.shape) != shape):
        raise ValueError(f"bias is {list(shape)} of {dtype}")


def matmul(a: Packed, b: Packed, dtype: torch.dtype = torch.bfloat16, bias: Optional[torch.Tensor] = None) -> torch.Tensor:
    """a b^T + bias for two matrices held in 8-bit integers."""
    _beside(a.cols, b)
    _kind(dtype, "dtype")
    _bias(bias, (b.rows,), dtype)
    g = _on(a.device, b.device, _device(bias))
    y = torch.empty(a.rows, b.rows, dtype=dtype, device=a.device)
    g.galv_i8_matmul(a.rows, 1, b.rows, a.cols, None, a.codes, a.scales, b.codes, b.scales, _vector(bias), (y.data_ptr(), b.rows), gb._DTYPES[dtype])
    return y


def linear(x: torch.Tensor, weight: Packed, bias: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x weight^T + bias over the last axis of x, put into 8-bit integers in the call, with weights held so; in x's type.  Without gradients."""
    dtype, shape = x.dtype, x.shape
    _kind(dtype, "x")
    if len(shape) < 1 or shape[-1] < 1:
        raise ValueError(f"x has a last axis of one number or more, not the shape {tuple(shape)}")
    _beside(shape[-1], weight)
    _bias(bias, (weight.rows,), dtype)
    device, n = x.device, weight.rows
    g = _on(device, weight.device, _device(bias))
    flat = _rows(x if len(shape) == 2 else x.reshape(-1, shape[-1]), "x")
    rows, cols = flat.shape
    y = torch.empty(rows, n, dtype=dtype, device=device)
    g.galv_i8_linear(rows, 1, n, cols, None, gb._matrix(flat), weight.codes, weight.scales, _vector(bias), (y.data_ptr(), n), gb._DTYPES[dtype], _bytes(_room(rows, cols), device))
    return y if len(shape) == 2 else y.view(*shape[:-1], n)
