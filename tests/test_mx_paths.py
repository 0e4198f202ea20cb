"""Microscaled operators: sizes that take each way through the kernels.

What a way has of its own (clusters, splits, segments, tiles after the first, launches ahead) is reached with numbers everywhere, and results are compared in
full.  Large products are compared with products of the held values in 64 bits on the device (torch), the others with numpy's.  Tolerances as in test_mx.
"""
import numpy as np
import pytest
import torch

from paper_2504_03662_b200 import mx

from .test_mx import DT, HALF, close, f64, numbers, packed, step

gpu = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------- products of few rows

@gpu
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("m,n,k", [(1, 1000, 4096), (16, 1000, 8192), (31, 2048, 4100), (64, 2300, 4096), (64, 130, 9000)])
def test_products_of_few_rows_in_clusters_of_eight(m, n, k, dtype):
    """At most 18 tiles of 128 columns and 16 chunks of 256 or more: eight CTAs share the summed index, some with two chunks each, and send their sums to one
    another."""
    (a, av), (b, bv) = packed(numbers(1, m, k, torch.float32), 4), packed(numbers(2, n, k, torch.float32), 4)
    bias = numbers(3, 1, n, DT[dtype])[0].cuda()
    want = av @ bv.T + f64(bias)
    tol = (k / 32 + 4) * 2 * HALF * (np.abs(av) @ np.abs(bv).T) + HALF * np.abs(want) + step(DT[dtype], want)
    first = mx.matmul(a, b, DT[dtype], bias)
    close(first, want, tol)
    for _ in range(20):
        assert torch.equal(mx.matmul(a, b, DT[dtype], bias), first)


# ------------------------------------------------------------------------------------------------- norms whose column sums a second kernel joins

def _norm_inputs(rows, cols, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, dy = (torch.randn(rows, cols, generator=g, device="cuda").to(dtype) for _ in range(2))
    return mx.pack(x), dy, (1 + torch.randn(cols, generator=g, device="cuda") / 10).to(dtype)


def _column_sums(kept, dy, kind, eps=1e-5):
    """(dweight, dbias, what dweight adds up, what dbias adds up) in 64 bits on the device."""
    x, y = mx.unpack(kept, torch.float32).double(), dy.double()
    c = x - x.mean(1, keepdim=True) if kind == "layer" else x
    r = 1 / (c.square().mean(1, keepdim=True) + eps).sqrt()
    terms = (y * c * r).abs().sum(0) + (y.abs() * x.abs().amax(1, keepdim=True) * r).sum(0)
    return (y * c * r).sum(0), y.sum(0), terms, y.abs().sum(0)


@gpu
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("rows,cols", [(2000, 64), (5000, 1000), (700, 5000), (300, 20000), (9, 70000)])
def test_joined_column_sums_captured_and_one_after_the_other(rows, cols, kind):
    """The join is launched ahead of the kernel before it.  Two norms in a row on one workspace, each followed at once by what reads its sums, eager and
    captured with new inputs at each replay: the same bits as alone, and the formula's sums."""
    galv = mx.context(torch.device("cuda", 0))
    need = galv.galv_mx_norm_workspace_bytes(rows, cols)
    assert need > 0
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")      # NaN where something is read that was not written
    sets = [_norm_inputs(rows, cols, torch.bfloat16, s) for s in range(4)]
    want = []
    for kept, dy, w in sets:
        _, dw, db = mx.norm_backward(dy, kept, w, kind)
        sw, sb, aw, ab = _column_sums(kept, dy, kind)
        # a term is off by 96 half steps, chains of additions by one half step of their magnitudes for each row at most
        assert ((dw.double() - sw).abs() <= (96 + rows) * HALF * aw).all()
        if kind == "layer":
            assert ((db.double() - sb).abs() <= (96 + rows) * HALF * ab).all()
        want.append(torch.stack([dw, db if kind == "layer" else torch.zeros_like(dw)]))
    static = [[(k.codes.clone(), k.scales.clone()), dy.clone(), w.clone()] for k, dy, w in sets[:2]]
    dx = torch.empty_like(static[0][1])
    dw, db = torch.empty(cols, device="cuda"), torch.zeros(cols, device="cuda")

    def both():
        out = []
        for (codes, scales), dy, w in static:
            galv.galv_mx_norm_backward(mx.NORMS[kind], 1e-5, codes, scales, dy, w, dx, dw, db if kind == "layer" else None, ws)
            out.append(torch.stack([dw, db]))
        return out

    assert all(torch.equal(a, b) for a, b in zip(both(), want[:2]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for first in (0, 2, 0, 2):
        for (held, dy, w), (kept, ndy, nw) in zip(static, sets[first:first + 2]):
            held[0].copy_(kept.codes), held[1].copy_(kept.scales), dy.copy_(ndy), w.copy_(nw)
        graph.replay()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, want[first:first + 2]))
