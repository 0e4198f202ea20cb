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
