"""Microscaled tensors: activations kept in 8 bits and used by the backward pass, products of operands in 4 bits.

A plan of the search says, layer by layer, what is kept and how fast the layer multiplies; the operators here carry the
microscaled choices out.  The functions allocate their results through PyTorch and call the library's kernels on the
current stream of the tensors' device; formats and formulas are those of include/galv.h.  `linear`, `norm` and
`activation` are the same as differentiable functions: their inputs are kept in 8 bits for the backward pass.

Calls and backward passes may be captured in a CUDA graph under PyTorch's rules: after the same call has run once on a
side stream, and for a backward pass with no eager graph of the same leaves alive.  Under autocast the differentiable functions compute in the types of
their inputs, as they do without.

A context of the library belongs to one host thread, so every thread (the autograd engine's among them) gets its own
for each device.

Waits inside the kernels of products are bounded (two seconds): those of `weight_grad` and `matmul` here and of all that modules i8 and experts have but `pack`, `unpack`
and `bias_grad`.  Where one has run out, the results since then are void: the next call of any of them on the device raises binding.GalvError with ERR_TIMEOUT, once in each thread, and so does
`check`, which waits for the current stream first (call it before results are relied on, and behind replays of captured graphs, which look at nothing).
"""
from __future__ import annotations

import threading
from typing import Optional, Union

import torch

from . import binding as gb

ACTS = {"gelu": gb.ACT_GELU, "gelu_tanh": gb.ACT_GELU_TANH, "silu": gb.ACT_SILU}
NORMS = {"layer": gb.NORM_LAYER, "rms": gb.NORM_RMS}
_NUMBERS = (torch.float32, torch.bfloat16, torch.float16)
_SHORT = (torch.bfloat16, torch.float16)
_local = threading.local()


def context(device: Union[int, torch.device]) -> gb.Galv:
    """This thread's library context on a CUDA device."""
    index = device if isinstance(device, int) else torch.cuda.current_device() if device.index is None else device.index
    try:
        return _local.made[index]
    except (AttributeError, KeyError):
        made = _local.__dict__.setdefault("made", {})
        made[index] = gb.Galv(index)
        return made[index]


def check(device: Union[int, torch.device]):
    """Waits for the current stream of a CUDA device; raises where a wait of a product has run out there since this thread's context was made or last looked."""
    context(device).galv_mx_status()


def codes_bytes(rows: int, cols: int, fmt: int = gb.MX8) -> int:
    return rows * ((cols + 31) // 32) * 4 * fmt


def scales_bytes(rows: int, cols: int, fmt: int = gb.MX8) -> int:
    nb = (cols + 31) // 32
    return rows * ((nb + 15) // 16 * 16) if fmt == gb.MX8 else (rows + 127) // 128 * ((nb + 3) // 4) * 512


class Packed:
    """A matrix [rows][cols] in blocks of 32 columns: element codes, one scale byte a block.  (What `pack` makes has both in one piece of memory, of
    which `codes` and `scales` are views made when they are asked for.)"""
    __slots__ = ("_codes", "_scales", "_both", "_at", "rows", "cols", "fmt", "device")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, rows: int, cols: int, fmt: int = gb.MX8):
        if fmt != gb.MX8 and fmt != gb.MX4:
            raise ValueError(f"a format is 8 or 4 bits, not {fmt}")
        if rows < 0 or cols < 1:
            raise ValueError(f"no matrix of {rows} rows and {cols} columns")
        nc, ns = codes_bytes(rows, cols, fmt), scales_bytes(rows, cols, fmt)
        if codes.dtype != torch.uint8 or scales.dtype != torch.uint8 or codes.numel() < nc or scales.numel() < ns or not codes.is_contiguous() or not scales.is_contiguous():
            raise ValueError(f"a [{rows}][{cols}] matrix in {fmt} bits takes {nc} and {ns} contiguous bytes, got {codes.dtype} {tuple(codes.shape)} and {scales.dtype} {tuple(scales.shape)}")
        if codes.device != scales.device:
            raise ValueError(f"codes on {codes.device} and scales on {scales.device}")
        self._codes, self._scales, self._both, self._at = codes, scales, None, (codes.data_ptr(), scales.data_ptr())
        self.rows, self.cols, self.fmt, self.device = rows, cols, fmt, codes.device

    @classmethod
    def _empty(cls, rows: int, cols: int, fmt: int, device: torch.device) -> "Packed":
        nc = (codes_bytes(rows, cols, fmt) + 255) & ~255
        p = cls.__new__(cls)
        p._codes = p._scales = None
        p._both = torch.empty(nc + scales_bytes(rows, cols, fmt), dtype=torch.uint8, device=device)
        at = p._both.data_ptr()
        p._at = at, at + nc
        p.rows, p.cols, p.fmt, p.device = rows, cols, fmt, device
        return p

    @property
    def codes(self) -> torch.Tensor:
        if self._codes is None:
            self._codes = self._both[:codes_bytes(self.rows, self.cols, self.fmt)]
        return self._codes

    @property
    def scales(self) -> torch.Tensor:
        if self._scales is None:
            self._scales = self._both[(codes_bytes(self.rows, self.cols, self.fmt) + 255) & ~255:]
        return self._scales

    @property
    def nbytes(self) -> int:
        return codes_bytes(self.rows, self.cols, self.fmt) + scales_bytes(self.rows, self.cols, self.fmt)


def _on(device: torch.device, *others: Optional[torch.device]) -> gb.Galv:
    """The context of the device that everything lies on."""
    for d in others:
        if d is not None and d != device:
            raise ValueError(f"operands on {device} and {d}")
    if device.type != "cuda":
        raise ValueError(f"microscaled operators take CUDA tensors (no CPU path), not {device.type}")
    return context(device.index)


def _device(t: Optional[torch.Tensor]) -> Optional[torch.device]:
    return None if t is None else t.device


def _kind(dtype: torch.dtype, what: str, dtypes=_NUMBERS):
    if dtype not in dtypes:
        raise ValueError(f"{what} is one of {', '.join(str(d).replace('torch.', '') for d in dtypes)}, not {dtype}")


def _rows(t: torch.Tensor, what: str) -> torch.Tensor:
    """A 2-D tensor whose rows are contiguous and do not overlap, and that lies in memory as it is (a copy where they are not, or it is a negative view)."""
    if t.is_neg():
        t = t.resolve_neg()
    if t.is_contiguous() and t.dim() == 2:
        return t
    if t.dim() != 2:
        raise ValueError(f"{what} is a matrix, not of shape {tuple(t.shape)}")
    if (t.shape[1] > 1 and t.stride(1) != 1) or (t.shape[0] > 1 and t.stride(0) < t.shape[1]):
        return t.contiguous()
    return t


def _vector(t: Optional[torch.Tensor]) -> Optional[torch.Tensor]:
    return None if t is None else t.resolve_neg().contiguous()


def _beside(t: torch.Tensor, p: Packed, what: str):
    if p.fmt != gb.MX8:
        raise ValueError("the backward pass reads what was kept in 8 bits")
    if t.shape[0] != p.rows or t.shape[1] != p.cols:
        raise ValueError(f"{what} of shape {tuple(t.shape)} beside a held matrix [{p.rows}][{p.cols}]")


def _bytes(n: int, device) -> torch.Tensor:
    return torch.empty(n, dtype=torch.uint8, device=device)


def pack(x: torch.Tensor, fmt: int = gb.MX8) -> Packed:
    """Holds a matrix in blocks of 8- or 4-bit elements."""
    if fmt != gb.MX8 and fmt != gb.MX4:
        raise ValueError(f"a format is 8 or 4 bits, not {fmt}")
    _kind(x.dtype, "x")
    x = _rows(x, "x")
    device = x.device
    g = _on(device)
    rows, cols = x.shape
    if cols < 1:
        raise ValueError("rows of at least one column")
    p = Packed._empty(rows, cols, fmt, device)
    g.galv_mx_pack(x, fmt, *p._at)
    return p


def unpack(p: Packed, dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """The numbers a packed matrix stands for."""
    _kind(dtype, "dtype")
    g = _on(p.device)
    x = torch.empty(p.rows, p.cols, dtype=dtype, device=p.device)
    g.galv_mx_unpack(p.fmt, *p._at, x)
    return x


def act_backward(dy: torch.Tensor, kept: Packed, act: str = "gelu") -> torch.Tensor:
    """dy * f'(x) for an activation function ("gelu", "gelu_tanh", "silu") whose input x was kept in 8 bits."""
    if act not in ACTS:
        raise ValueError(f"an activation function is one of {', '.join(ACTS)}, not {act!r}")
    _kind(dy.dtype, "dy")
    dy = _rows(dy, "dy")
    _beside(dy, kept, "dy")
    device = dy.device
    g = _on(device, kept.device)
    dx = torch.empty(kept.rows, kept.cols, dtype=dy.dtype, device=device)
    g.galv_mx_act_backward(ACTS[act], *kept._at, dy, dx)
    return dx


def norm_backward(dy: torch.Tensor, kept: Packed, weight: Optional[torch.Tensor] = None, kind: str = "layer", eps: float = 1e-5):
    """(dx, dweight, dbias) of a "layer" or "rms" norm over rows whose input was kept in 8 bits; dweight and dbias in fp32, dbias None for "rms"."""
    if kind not in NORMS:
        raise ValueError(f"a norm is one of {', '.join(NORMS)}, not {kind!r}")
    _kind(dy.dtype, "dy")
    dy = _rows(dy, "dy")
    _beside(dy, kept, "dy")
    if weight is not None and (weight.dtype != dy.dtype or tuple(weight.shape) != (kept.cols,)):
        raise ValueError(f"weight is [{kept.cols}] of {dy.dtype}")
    device = dy.device
    g = _on(device, kept.device, _device(weight))
    dx = torch.empty(kept.rows, kept.cols, dtype=dy.dtype, device=device)
    dweight = torch.empty(kept.cols, dtype=torch.float32, device=device)
    dbias = torch.empty(kept.cols, dtype=torch.float32, device=device) if kind == "layer" else None
    n = g.galv_mx_norm_workspace_bytes(kept.rows, kept.cols)
    g.galv_mx_norm_backward(NORMS[kind], eps, *kept._at, dy, _vector(weight), dx, dweight, dbias, _bytes(n, device) if n else None)
    return dx, dweight, dbias


def weight_grad(dy: torch.Tensor, kept: Packed, dtype: Optional[torch.dtype] = None, base: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """base + dy^T x for a linear layer whose input x was kept in 8 bits: [columns of dy][columns of x].  `out` may be `base`."""
    _kind(dy.dtype, "dy", _SHORT)
    dy = _rows(dy, "dy")
    if kept.fmt != gb.MX8:
        raise ValueError("the backward pass reads what was kept in 8 bits")
    if dy.shape[0] != kept.rows or dy.shape[1] < 1:
        raise ValueError(f"dy of shape {tuple(dy.shape)} beside {kept.rows} kept rows")
    shape = (dy.shape[1], kept.cols)
    dtype = dtype or (out if out is not None else base if base is not None else dy).dtype
    if dtype != dy.dtype and dtype != torch.float32:
        raise ValueError(f"a weight gradient is of {dy.dtype} or float32, not {dtype}")
    for t, what in ((base, "base"), (out, "out")):
        if t is not None:
            if t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous() or t.is_neg():
                raise ValueError(f"{what} is a contiguous {shape} of {dtype}")
    device = dy.device
    g = _on(device, kept.device, _device(base), _device(out))
    dw = torch.empty(shape, dtype=dtype, device=device) if out is None else out
    n = g.galv_mx_weight_grad_workspace_bytes(dy, kept.cols)
    g.galv_mx_weight_grad(dy, *kept._at, base, dw, _bytes(n, device) if n else None)
    return dw


def matmul(a: Packed, b: Packed, dtype: torch.dtype = torch.bfloat16, bias: Optional[torch.Tensor] = None) -> torch.Tensor:
    """a b^T + bias for two matrices held in 4 bits."""
    if a.fmt != gb.MX4 or b.fmt != gb.MX4:
        raise ValueError("a product takes operands held in 4 bits")
    if a.cols != b.cols or b.rows < 1:
        raise ValueError(f"a product of [{a.rows}][{a.cols}] and [{b.rows}][{b.cols}] transposed")
    _kind(dtype, "dtype")
    if bias is not None and (bias.dtype != dtype or tuple(bias.shape) != (b.rows,)):
        raise ValueError(f"bias is [{b.rows}] of {dtype}")
    g = _on(a.device, b.device, _device(bias))
    y = torch.empty(a.rows, b.rows, dtype=dtype, device=a.device)
    n = g.galv_mx_matmul_workspace_bytes(a.rows, b.rows, a.cols)
    g.galv_mx_matmul(a.cols, *a._at, *b._at, _vector(bias), y, _bytes(n, a.device) if n else None)
    return y


# ------------------------------------------------------------------------------------------------- differentiable forms

def _flat(x: torch.Tensor) -> torch.Tensor:
    return x.reshape(-1, x.shape[-1])


def _last_axis(x: torch.Tensor):
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError(f"x has a last axis of one number or more, not the shape {tuple(x.shape)}")


def _as_typed(f):
    """A forward or backward pass in the types of its inputs: under autocast the library's norms would answer in fp32, its products in autocast's type."""
    def run(*args):
        if torch.is_autocast_enabled("cuda"):
            with torch.autocast("cuda", enabled=False):
                return f(*args)
        return f(*args)
    return run


class _Linear(torch.autograd.Function):
    @staticmethod
    @_as_typed
    def forward(ctx, x, weight, bias, four, keep, eight):
        flat = _flat(x)
        if four:
            y = matmul(pack(flat, gb.MX4), pack(weight, gb.MX4), x.dtype, bias)
        elif eight:
            from . import i8                              # which takes its checks from this module
            y = i8.linear(flat, i8.pack(weight), bias)
        else:
            y = flat @ weight.t() if bias is None else torch.addmm(bias, flat, weight.t())
        kept = pack(flat) if keep and ctx.needs_input_grad[1] else None
        ctx.save_for_backward(weight, *((kept.codes, kept.scales) if kept else ()))
        ctx.shape, ctx.has_bias = x.shape, bias is not None
        return y.view(*x.shape[:-1], weight.shape[0])

    @staticmethod
    @torch.autograd.function.once_differentiable
    @_as_typed
    def backward(ctx, dy):
        weight, *kept = ctx.saved_tensors
        flat = _flat(dy)
        dx = dw = db = None
        if ctx.needs_input_grad[0]:
            dx = (flat @ weight).view(ctx.shape)
        if ctx.needs_input_grad[1]:
            dw = weight_grad(flat, Packed(*kept, flat.shape[0], weight.shape[1]), weight.dtype)
        if ctx.has_bias and ctx.needs_input_grad[2]:
            db = flat.sum(0, dtype=torch.float32).to(dy.dtype)
        return dx, dw, db, None, None, None


def linear(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, four: bool = False, eight: bool = False) -> torch.Tensor:
    """x weight^T + bias (bf16 or fp16), x kept in 8 bits for the weight's gradient (where one will be taken).  `four`: the forward product takes both operands in
    4 bits; `eight`: in 8-bit integers with a scale for each token and each output (module i8); the gradients are those of the product of the unrounded operands (straight
    through the rounding)."""
    _kind(x.dtype, "x", _SHORT)
    _last_axis(x)
    if weight.dim() != 2 or weight.dtype != x.dtype or weight.shape[0] < 1 or weight.shape[1] != x.shape[-1]:
        raise ValueError(f"weight of shape {tuple(weight.shape)} and {weight.dtype} beside x of {tuple(x.shape)} and {x.dtype}")
    if bias is not None and (bias.dtype != x.dtype or bias.dim() > 1):
        raise ValueError(f"bias is [{weight.shape[0]}] of {x.dtype}, not {tuple(bias.shape)} of {bias.dtype}")
    if eight:
        if four:
            raise ValueError("a forward product is in 4 bits or in 8-bit integers, not both")
        if x.shape[-1] > gb.I8_MOST:
            raise ValueError(f"products of 8-bit integers sum up to {gb.I8_MOST} columns, not {x.shape[-1]}")
        if bias is not None and tuple(bias.shape) != weight.shape[:1]:
            raise ValueError(f"bias is [{weight.shape[0]}] of {x.dtype}, not {tuple(bias.shape)} of {bias.dtype}")
    return _Linear.apply(x, weight, bias, four, torch.is_grad_enabled(), eight)


class _Norm(torch.autograd.Function):
    @staticmethod
    @_as_typed
    def forward(ctx, x, weight, bias, kind, eps, keep):
        n = (x.shape[-1],)
        y = torch.nn.functional.layer_norm(x, n, weight, bias, eps) if kind == "layer" else torch.nn.functional.rms_norm(x, n, weight, eps)
        if keep and any(ctx.needs_input_grad):
            kept = pack(_flat(x))
            ctx.save_for_backward(kept.codes, kept.scales, *(() if weight is None else (weight,)))
            ctx.kind, ctx.eps, ctx.shape, ctx.bias_type = kind, eps, x.shape, None if bias is None else bias.dtype
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    @_as_typed
    def backward(ctx, dy):
        codes, scales, *weight = ctx.saved_tensors
        flat = _flat(dy)
        dx, dw, db = norm_backward(flat, Packed(codes, scales, *flat.shape), weight[0] if weight else None, ctx.kind, ctx.eps)
        return (dx.view(ctx.shape), dw.to(weight[0].dtype) if weight else None, None if ctx.bias_type is None else db.to(ctx.bias_type), None, None, None)


def norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, kind: str = "layer", eps: float = 1e-5) -> torch.Tensor:
    """A "layer" or "rms" norm over the last axis, x kept in 8 bits for the backward pass (where there will be one)."""
    if kind not in NORMS:
        raise ValueError(f"a norm is one of {', '.join(NORMS)}, not {kind!r}")
    if kind == "rms" and bias is not None:
        raise ValueError("an rms norm has no bias")
    if not eps >= 0:
        raise ValueError(f"eps is 0 or more, not {eps}")
    _kind(x.dtype, "x")
    _last_axis(x)
    for t, what in ((weight, "weight"), (bias, "bias")):
        if t is not None and (t.dtype != x.dtype or tuple(t.shape) != x.shape[-1:]):
            raise ValueError(f"{what} is [{x.shape[-1]}] of {x.dtype}")
    _on(x.device, _device(weight), _device(bias))
    return _Norm.apply(x, weight, bias, kind, eps, torch.is_grad_enabled())


class _Activation(torch.autograd.Function):
    @staticmethod
    @_as_typed
    def forward(ctx, x, act, keep):
        if keep and ctx.needs_input_grad[0]:
            kept = pack(_flat(x))
            ctx.save_for_backward(kept.codes, kept.scales)
            ctx.act, ctx.shape = act, x.shape
        f = torch.nn.functional
        return f.silu(x) if act == "silu" else f.gelu(x, approximate="tanh" if act == "gelu_tanh" else "none")

    @staticmethod
    @torch.autograd.function.once_differentiable
    @_as_typed
    def backward(ctx, dy):
        flat = _flat(dy)
        return act_backward(flat, Packed(*ctx.saved_tensors, *flat.shape), ctx.act).view(ctx.shape), None, None


def activation(x: torch.Tensor, act: str = "gelu") -> torch.Tensor:
    """gelu, gelu_tanh or silu, x kept in 8 bits for the backward pass (where there will be one)."""
    if act not in ACTS:
        raise ValueError(f"an activation function is one of {', '.join(ACTS)}, not {act!r}")
    _kind(x.dtype, "x")
    _last_axis(x)
    _on(x.device)
    return _Activation.apply(x, act, torch.is_grad_enabled())
