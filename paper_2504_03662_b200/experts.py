"""Products of rows by their expert's weights: layers whose weights are chosen row by row.

The rows of x are sorted by expert and `ends` (int32, one an expert, on the device) says where each expert's rows end: counts.cumsum(0, dtype=torch.int32).
It is read by the kernels alone, so nothing waits for it and calls may be captured.  Ends that fall or leave the rows count as clamped; rows from the last end on
belong to no expert: their results are zeros, and they enter no gradient, whatever they hold.  At most 1024 experts.

The functions allocate their results through PyTorch and call the library's kernels on the current stream of the tensors' device; formulas are those of
include/galv.h.  `linear` is the same as a differentiable function.  Captures in CUDA graphs, contexts and waits that have run out: as in mx.
"""
from __future__ import annotations

from typing import Optional, Union

import torch

from . import binding as gb, i8
from .mx import _SHORT, _as_typed, _bytes, _device, _kind, _on, _rows


def _ends(ends: torch.Tensor, experts: int):
    if ends.dtype != torch.int32 or tuple(ends.shape) != (experts,):
        raise ValueError(f"ends is [{experts}] of int32, not {tuple(ends.shape)} of {ends.dtype}")


def _count(experts: int):
    if not 1 <= experts <= gb.EXPERTS_MOST:
        raise ValueError(f"1 to {gb.EXPERTS_MOST} experts, not {experts}")


def _whole(t: Optional[torch.Tensor]) -> Optional[torch.Tensor]:
    """As it lies in memory, without gaps."""
    return t if t is None or (t.is_contiguous() and not t.is_neg()) else t.detach().resolve_neg().contiguous()


def _apart(weight: torch.Tensor) -> torch.Tensor:
    """Weights whose rows are contiguous and one distance apart (a copy where they are not): rows kept on 16-byte boundaries are used as they lie."""
    if weight.is_contiguous() and not weight.is_neg():
        return weight
    experts, n, k = weight.shape
    first, stride, step = weight.stride()
    if weight.is_neg() or step != 1 or stride < k or first != n * stride or n == 1:
        return _whole(weight)
    return weight


def _weight(weight: torch.Tensor, dtype: torch.dtype):
    if weight.dim() != 3 or weight.dtype != dtype or weight.shape[1] < 1 or weight.shape[2] < 1:
        raise ValueError(f"weight is [experts][columns of y][columns of x] of {dtype}, not {tuple(weight.shape)} of {weight.dtype}")
    _count(weight.shape[0])


def _products(x: torch.Tensor, weight: i8.Packed, ends: torch.Tensor, bias, dtype: torch.dtype) -> torch.Tensor:
    """Experts' weights in 8-bit integers, stacked along their rows."""
    if ends.dim() != 1:
        raise ValueError(f"ends is [experts] of int32, not {tuple(ends.shape)} of {ends.dtype}")
    experts = ends.shape[0]
    _ends(ends, experts)
    _count(experts)
    if weight.rows % experts:
        raise ValueError(f"weights of {experts} experts in {weight.rows} rows")
    n, held = weight.rows // experts, isinstance(x, i8.Packed)
    rows, cols = (x.rows, x.cols) if held else x.shape
    i8._beside(cols, weight)
    i8._bias(bias, (experts, n), dtype)
    device = x.device
    g = _on(device, weight.device, ends.device, _device(bias))
    y = torch.empty(rows, n, dtype=dtype, device=device)
    out, number = (y.data_ptr(), n), gb._DTYPES[dtype]
    if held:
        g.galv_i8_matmul(rows, experts, n, cols, _whole(ends), x.codes, x.scales, weight.codes, weight.scales, _whole(bias), out, number)
    else:
        g.galv_i8_linear(rows, experts, n, cols, _whole(ends), gb._matrix(x), weight.codes, weight.scales, _whole(bias), out, number, _bytes(i8._room(rows, cols), device))
    return y


def matmul(x: Union[torch.Tensor, i8.Packed], weight: Union[torch.Tensor, i8.Packed], ends: torch.Tensor, bias: Optional[torch.Tensor] = None,
           dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """x weight[e]^T + bias[e] for each row of x and its expert e.  Without gradients (`linear` has them).

    weight [experts][columns of y][columns of x] and x [rows][columns] in 16 bits; or weights held in 8-bit integers with the experts' rows one behind the
    other, and x in numbers, which are put into 8-bit integers in the call, or held so too.  bias [experts][columns of y] of y's type: x's, or `dtype` where x is held.
    """
    if isinstance(x, i8.Packed):
        if not isinstance(weight, i8.Packed):
            raise ValueError("rows held in 8-bit integers are multiplied by weights held so")
        dtype = dtype or torch.bfloat16
        _kind(dtype, "dtype")
        return _products(x, weight, ends, bias, dtype)
    if dtype is not None and dtype != x.dtype:
        raise ValueError(f"y is of x's type {x.dtype}, not {dtype}")
    if isinstance(weight, i8.Packed):
        _kind(x.dtype, "x")
        return _products(_rows(x, "x"), weight, ends, bias, x.dtype)
    return _forward(x, weight, ends, bias)[0]


def _forward(x: torch.Tensor, weight: torch.Tensor, ends: torch.Tensor, bias: Optional[torch.Tensor]):
    """y, and what was multiplied: x and weight as they lie, and the workspace in which the library has moved either to 16-byte boundaries."""
    dtype, device, shape = x.dtype, x.device, weight.shape
    _kind(dtype, "x", _SHORT)
    _weight(weight, dtype)
    experts, n, k = shape
    _ends(ends, experts)
    x = _rows(x, "x")
    rows, cols = x.shape
    if cols != k:
        raise ValueError(f"x of shape {tuple(x.shape)} beside weights of {k} columns")
    i8._bias(bias, (experts, n), dtype)
    g = _on(device, weight.device, ends.device, _device(bias))
    y = torch.empty(rows, n, dtype=dtype, device=device)
    weight, ends = _apart(weight), _whole(ends)
    xm, wm = gb._matrix(x), gb._matrices(weight)
    ws = None
    if not _lie(n, xm, wm):
        size = g.galv_expert_matmul_workspace_bytes(rows, experts, n, k, xm, wm)
        ws = _bytes(size, device) if size else None
    g.galv_expert_matmul(rows, experts, n, k, ends, xm, wm, _whole(bias), (y.data_ptr(), n), gb._DTYPES[dtype], ws)
    return y, x, weight, ends, ws


def _lie(n: int, *matrices) -> bool:
    """Whether rows start on 16-byte boundaries, nearer to one another than the header's limit: then the library moves nothing."""
    for start, stride in matrices:
        if start and (start % 16 or stride % 8 or n * stride >= 1 << 39):
            return False
    return True


def _moved(x: torch.Tensor, weight: torch.Tensor, ws: Optional[torch.Tensor]):
    """Of a forward product: x and weight on 16-byte boundaries, where they were moved to such in its workspace, else as they are."""
    if ws is None:
        return x, weight
    (rows, k), (experts, n, _) = x.shape, weight.shape
    pitch, at, both = gb.load_library().galv_expert_pitch(k), 0, ws.view(x.dtype)
    start, stride = gb._matrix(x)
    if start % 16 or stride % 8 or stride >= 1 << 39:
        x, at = both.as_strided((rows, k), (pitch, 1)), (rows * pitch * 2 + 255 & ~255) // 2
    if at < both.numel():
        weight = both.as_strided((experts, n, k), (n * pitch, pitch, 1), at)
    return x, weight


def input_grad(dy: torch.Tensor, weight: torch.Tensor, ends: torch.Tensor) -> torch.Tensor:
    """dy weight[e] for each row of dy and its expert e: the gradient of x."""
    _kind(dy.dtype, "dy", _SHORT)
    _weight(weight, dy.dtype)
    experts, n, k = weight.shape
    _ends(ends, experts)
    dy = _rows(dy, "dy")
    if dy.shape[1] != n:
        raise ValueError(f"dy of shape {tuple(dy.shape)} beside weights of {n} rows")
    g = _on(dy.device, weight.device, ends.device)
    dx = torch.empty(dy.shape[0], k, dtype=dy.dtype, device=dy.device)
    weight = _apart(weight)
    size = g.galv_expert_input_grad_workspace_bytes(dy, weight)
    g.galv_expert_input_grad(_whole(ends), dy, weight, dx, _bytes(size, dy.device) if size else None)
    return dx


def weight_grad(dy: torch.Tensor, x: torch.Tensor, ends: torch.Tensor, dtype: Optional[torch.dtype] = None, base: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """base[e] + dy^T x over the rows of each expert e: [experts][columns of dy][columns of x].  `out` may be `base`."""
    _kind(dy.dtype, "dy", _SHORT)
    if ends.dim() != 1:
        raise ValueError(f"ends is [experts] of int32, not {tuple(ends.shape)} of {ends.dtype}")
    experts = ends.shape[0]
    _ends(ends, experts)
    _count(experts)
    dy, x = _rows(dy, "dy"), _rows(x, "x")
    if x.dtype != dy.dtype or x.shape[0] != dy.shape[0] or x.shape[1] < 1 or dy.shape[1] < 1:
        raise ValueError(f"dy of shape {tuple(dy.shape)} and {dy.dtype} beside x of {tuple(x.shape)} and {x.dtype}")
    shape = (experts, dy.shape[1], x.shape[1])
    dtype = dtype or (out if out is not None else base if base is not None else dy).dtype
    if dtype != dy.dtype and dtype != torch.float32:
        raise ValueError(f"a weight gradient is of {dy.dtype} or float32, not {dtype}")
    for t, what in ((base, "base"), (out, "out")):
        if t is not None:
            if t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous() or t.is_neg():
                raise ValueError(f"{what} is a contiguous {shape} of {dtype}")
    g = _on(dy.device, x.device, ends.device, _device(base), _device(out))
    dw = torch.empty(shape, dtype=dtype, device=dy.device) if out is None else out
    size = g.galv_expert_weight_grad_workspace_bytes(experts, dy, x)
    g.galv_expert_weight_grad(_whole(ends), dy, x, base, dw, _bytes(size, dy.device) if size else None)
    return dw


def bias_grad(dy: torch.Tensor, ends: torch.Tensor, dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """The sum of dy over the rows of each expert: [experts][columns of dy], in dy's type or float32."""
    _kind(dy.dtype, "dy", _SHORT)
    if ends.dim() != 1:
        raise ValueError(f"ends is [experts] of int32, not {tuple(ends.shape)} of {ends.dtype}")
    _ends(ends, ends.shape[0])
    _count(ends.shape[0])
    dy = _rows(dy, "dy")
    dtype = dtype or dy.dtype
    if dy.shape[1] < 1 or (dtype != dy.dtype and dtype != torch.float32):
        raise ValueError(f"sums of dy of shape {tuple(dy.shape)} in {dy.dtype} or float32, not {dtype}")
    g = _on(dy.device, ends.device)
    db = torch.empty(ends.shape[0], dy.shape[1], dtype=dtype, device=dy.device)
    g.galv_expert_bias_grad(_whole(ends), dy, db)
    return db


class _Linear(torch.autograd.Function):
    @staticmethod
    @_as_typed
    def forward(ctx, x, weight, ends, bias):
        y, x, weight, ends, ws = _forward(x, weight, ends, bias)
        need_x, need_w, _, _ = ctx.needs_input_grad
        if ws is not None:
            x, weight = _moved(x, weight, ws)             # the backward pass need not move them again
        ctx.save_for_backward(x if need_w else None, weight if need_x else None, ends)
        ctx.shape = weight.shape
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    @_as_typed
    def backward(ctx, dy):
        x, weight, ends = ctx.saved_tensors               # as they lie, from the forward pass
        need_x, need_w, _, need_b = ctx.needs_input_grad
        experts, n, k = ctx.shape
        dy = _rows(dy, "dy")
        rows, dtype, device = dy.shape[0], dy.dtype, dy.device
        dx = torch.empty(rows, k, dtype=dtype, device=device) if need_x else None
        dw = torch.empty(experts, n, k, dtype=dtype, device=device) if need_w else None
        db = torch.empty(experts, n, dtype=dtype, device=device) if need_b else None
        g = _on(device)
        dm, xm, wm = gb._matrix(dy), gb._matrix(x) if need_w else (None, 0), gb._matrices(weight)
        ws = None
        if need_w or not _lie(n, dm, xm, wm):             # weight gradients may keep sums of parts of their rows there: the library says so
            size = g.galv_expert_backward_workspace_bytes(rows, experts, n, k, dm, xm, wm)
            ws = _bytes(size, device) if size else None
        g.galv_expert_backward(rows, experts, n, k, ends, dm, xm, wm, gb._DTYPES[dtype], (dx.data_ptr(), k) if need_x else (None, 0), dw, db, ws)
        return dx, dw, None, db


def linear(x: torch.Tensor, weight: torch.Tensor, ends: torch.Tensor, bias: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x weight[e]^T + bias[e] for each row of x and its expert e, in 16 bits, with gradients for x, weight and bias (where they are taken).  Of operands whose rows do not start
    on 16-byte boundaries the copies that the forward product takes are kept for the backward pass: 2 bytes for each element and what fills its rows up, of the weights as much as they take
    themselves, unless they are kept with rows further apart (weight.stride(1) and its start multiples of 8 elements)."""
    return _Linear.apply(x, weight, ends, bias)
