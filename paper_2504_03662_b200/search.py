"""Device buffers for one workload and the calls that run the path on them.

Holds no arithmetic: tensors are allocated through PyTorch and handed to the C
library; every step (cost model, validation, recurrence, optimum, backtrack)
runs in the library's kernels.
"""
from __future__ import annotations

from typing import Optional

import numpy as np
import torch

from . import binding as gb, mx
from .inputs import FORM_DESC, Workload


def _dev_bytes(a: np.ndarray, device) -> torch.Tensor:
    return torch.from_numpy(np.ascontiguousarray(a).view(np.uint8).reshape(-1).copy()).to(device)


def _seconds(f, reps: int = 5) -> float:
    """Shortest time of a call on the current stream, by events, after two calls that are not timed."""
    best = float("inf")
    for k in range(reps + 2):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        f()
        b.record()
        b.synchronize()
        if k >= 2:
            best = min(best, a.elapsed_time(b) * 1e-3)
    return best


def measure_forms(galv: gb.Galv, hidden: int, tokens: int, keep: bool = True, multiply: bool = True) -> np.ndarray:
    """Forms of strategies (rows of FORM_DESC for Workload.with_forms) with the rates of this device: the hardware profiler's part for the
    microscaled operators.  A layer's input [tokens][hidden] in bf16 is packed in 8 bits and used in the backward pass, beside the plain backward pass of
    the 16-bit input: the dearest of what may read it counts (the gradient of a weight, of a norm, of an activation function, or restoring it, as
    queries, keys, values and checkpointed inputs are); and multiplied in 4 bits by a weight [hidden][hidden] (both packed in the call, as mx.linear does it), beside the plain
    product.  These are rates of one shape: layers of very different widths want their own."""
    if hidden < 1 or tokens < 1:
        raise ValueError(f"rates of a layer of {tokens} tokens x {hidden}: both are at least 1")
    dev = torch.device("cuda", galv.device)
    g = torch.Generator(device=dev).manual_seed(1)
    x, dy, w = (torch.randn(*s, generator=g, device=dev).to(torch.bfloat16) for s in ((tokens, hidden), (tokens, hidden), (hidden, hidden)))
    rows = []
    s_per_byte, speed = 0.0, 1.0
    with torch.cuda.device(dev):
        if keep:
            kept = mx.pack(x)
            ops, ones = torch.ops.aten, torch.ones(hidden, dtype=x.dtype, device=dev)
            stats = ops.native_layer_norm(x, [hidden], ones, ones, 1e-5)[1:]
            uses = [(lambda: mx.weight_grad(dy, kept), lambda: dy.t() @ x),
                    (lambda: mx.norm_backward(dy, kept, ones), lambda: ops.native_layer_norm_backward(dy, x, [hidden], *stats, ones, ones, [True] * 3)),
                    (lambda: mx.act_backward(dy, kept), lambda: ops.gelu_backward(dy, x))]
            more = [_seconds(held) - _seconds(plain) for held, plain in uses] + [_seconds(lambda: mx.unpack(kept))]
            s_per_byte = (_seconds(lambda: mx.pack(x)) + max(more)) / (x.numel() * 2)
            rows.append((8, 0, s_per_byte, 1.0))
        if multiply:
            speed = _seconds(lambda: x @ w.t()) / _seconds(lambda: mx.matmul(mx.pack(x, gb.MX4), mx.pack(w, gb.MX4)))
            rows.append((0, 4, 0.0, speed))
        if keep and multiply:
            rows.append((8, 4, s_per_byte, speed))
    return np.array(rows, FORM_DESC)


class SearchBuffers:
    """All device arrays of one batch, laid out as the C boundary expects."""

    def __init__(self, galv: gb.Galv, w: Workload, flags: int = gb.STORE_C_FULL, device: Optional[str] = None):
        self.galv, self.w, self.flags = galv, w, flags
        dev = torch.device(device or f"cuda:{galv.device}")
        self.dev = dev
        if w.trans_q is not None and w.trans_q.ndim == 4:          # one transition matrix per layer
            flags |= gb.TRANS_PER_LAYER
        self.flags = flags
        self.shape = gb.make_shape(w.B, w.Lmax, w.S, w.M, flags)
        B, Lm, S, P = w.B, w.Lmax, w.S, self.shape.m_pitch
        i32 = dict(dtype=torch.int32, device=dev)
        self.L = torch.from_numpy(np.ascontiguousarray(w.L, np.int32)).to(dev)
        if w.has_model:
            self.layers = _dev_bytes(w.layers, dev)
            self.layer_stride_B = 0 if w.layers.shape[0] == 1 else w.Lmax
            self.strat = _dev_bytes(w.strat, dev)
            self.inst = _dev_bytes(w.inst, dev)
            self.time_q = torch.zeros(B, Lm, S, **i32)
            self.mem_q = torch.zeros(B, Lm, S, **i32)
            self.trans_q = torch.zeros(B, S, S, **i32)
        else:
            self.time_q = torch.from_numpy(np.ascontiguousarray(w.time_q, np.int32)).to(dev)
            self.mem_q = torch.from_numpy(np.ascontiguousarray(w.mem_q, np.int32)).to(dev)
            self.trans_q = torch.from_numpy(np.ascontiguousarray(w.trans_q, np.int32)).to(dev)
        self.time_s = self.mem_bytes = self.forms = None
        if w.forms is not None:
            self.forms = _dev_bytes(w.forms, dev)
            self.form_layers = self.layers if w.masks is None else _dev_bytes(w.form_layers, dev)
        self.C = torch.empty(B, Lm, S, P, **i32) if flags & gb.STORE_C_FULL else None
        self.A = torch.empty(B, Lm, S, P, dtype=torch.uint8, device=dev) if flags & gb.STORE_ARGMIN else None
        self.C_last = torch.empty(B, S, P, **i32)
        self.workspace = torch.empty(max(256, galv.galv_dp_workspace_bytes(self.shape)), dtype=torch.uint8, device=dev)
        self.status = torch.zeros(B, **i32)
        self.opt_cost = torch.empty(B, **i32)
        self.plan = torch.full((B, Lm), -1, **i32)             # stays -1 / 0 when no table is kept (cost-only search)
        self.mem_used = torch.zeros(B, **i32)

    def eval_costs(self, want_fp64: bool = False):
        w = self.w
        assert w.has_model
        want_fp64 = want_fp64 or self.forms is not None            # forms are priced from the doubles
        if want_fp64 and self.time_s is None:
            self.time_s = torch.zeros(w.B, w.Lmax, w.S, dtype=torch.float64, device=self.dev)
            self.mem_bytes = torch.zeros(w.B, w.Lmax, w.S, dtype=torch.float64, device=self.dev)
        self.galv.galv_eval_costs(self.shape, self.L, self.layers, self.layer_stride_B, self.strat, self.inst,
                                  self.time_s if want_fp64 else None, self.mem_bytes if want_fp64 else None,
                                  self.time_q, self.mem_q, self.trans_q, self.status)
        if self.forms is not None:
            self.galv.galv_add_form_cost(self.shape, self.L, self.form_layers, self.layer_stride_B, self.strat, self.inst, self.forms,
                                         self.time_s, self.mem_bytes, self.time_q, self.mem_q)

    def dp_search(self):
        self.galv.galv_dp_search(self.shape, self.L, self.time_q, self.mem_q, self.trans_q, self.C, self.A,
                                 self.C_last, self.workspace, self.status)

    def backtrack(self, budget: Optional[torch.Tensor] = None, use_A: Optional[bool] = None):
        A = self.A if (use_A is None or use_A) else None
        C = self.C if (use_A is None or not use_A) else None
        walk = C is not None or A is not None                   # a plan needs one of the tables
        self.galv.galv_backtrack(self.shape, self.L, self.time_q, self.mem_q, self.trans_q, C, A, self.C_last,
                                 budget, self.opt_cost, self.plan if walk else None, self.mem_used if walk else None,
                                 self.status)

    def step(self):
        """One pass of the whole path on the current stream (asynchronous)."""
        if self.w.has_model:
            self.eval_costs()
        self.dp_search()
        self.backtrack()

    def results(self):
        torch.cuda.synchronize(self.dev)
        return dict(opt_cost=self.opt_cost.cpu().numpy(), plan=self.plan.cpu().numpy(),
                    mem_used=self.mem_used.cpu().numpy(), status=self.status.cpu().numpy())

    def table(self, i: int) -> np.ndarray:
        """C of instance i in the recurrence's index order [L][M+1][S] (host copy)."""
        M = self.w.M
        return np.ascontiguousarray(self.C[i, :, :, :M + 1].permute(0, 2, 1).cpu().numpy())

    def argmin_table(self, i: int) -> np.ndarray:
        M = self.w.M
        return np.ascontiguousarray(self.A[i, :, :, :M + 1].permute(0, 2, 1).cpu().numpy())


class HostSearch:
    """The host-buffer entry point: pinned host inputs/outputs and a device arena."""

    def __init__(self, galv: gb.Galv, w: Workload, flags: int = gb.STORE_C_FULL):
        if w.forms is not None:
            raise ValueError("the host entry point prices no forms: use SearchBuffers")
        self.galv, self.w = galv, w
        if w.trans_q is not None and w.trans_q.ndim == 4:          # one transition matrix per layer
            flags |= gb.TRANS_PER_LAYER
        self.shape = gb.make_shape(w.B, w.Lmax, w.S, w.M, flags)
        pin = lambda a: torch.from_numpy(np.ascontiguousarray(a).view(np.uint8).reshape(-1).copy()).pin_memory()
        self.L = pin(np.ascontiguousarray(w.L, np.int32))
        self.model = w.has_model
        if self.model:
            self.layers, self.strat, self.inst = pin(w.layers), pin(w.strat), pin(w.inst)
            self.layer_stride_B = 0 if w.layers.shape[0] == 1 else w.Lmax
            self.tq = self.mq = self.xq = None
            self.h2d = sum(t.numel() for t in (self.L, self.layers, self.strat, self.inst))
        else:
            self.layers = self.strat = self.inst = None
            self.layer_stride_B = 0
            self.tq, self.mq, self.xq = pin(w.time_q), pin(w.mem_q), pin(w.trans_q)
            self.h2d = sum(t.numel() for t in (self.L, self.tq, self.mq, self.xq))
        i32 = dict(dtype=torch.int32)
        self.opt_cost = torch.empty(w.B, **i32).pin_memory()
        self.plan = torch.empty(w.B, w.Lmax, **i32).pin_memory()
        self.mem_used = torch.empty(w.B, **i32).pin_memory()
        self.status = torch.empty(w.B, **i32).pin_memory()
        self.d2h = 4 * (3 * w.B + w.B * w.Lmax)
        self.arena = torch.empty(galv.galv_search_host_arena_bytes(self.shape, self.model), dtype=torch.uint8,
                                 device=f"cuda:{galv.device}")

    def run(self):
        """Synchronous: returns when the results are in the host buffers."""
        self.galv.galv_search_host(self.shape, self.L, self.layers, self.layer_stride_B, self.strat, self.inst,
                                   self.tq, self.mq, self.xq, self.opt_cost, self.plan, self.mem_used, self.status,
                                   self.arena)
        return dict(opt_cost=self.opt_cost.numpy(), plan=self.plan.numpy(), mem_used=self.mem_used.numpy(),
                    status=self.status.numpy())
