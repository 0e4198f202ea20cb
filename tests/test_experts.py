"""Products of rows by their expert's weights, and their gradients.

The references are the formulas in 64 bits, expert by expert.  Tolerances count roundings: half a step of the output's type, and 2^-23 of the magnitudes that are
summed for each step of 16 that a tensor core adds (it may cut instead of round), 2^-24 for each addition in fp32.
"""
import numpy as np
import pytest
import torch

from paper_2504_03662_b200 import binding as gb
from paper_2504_03662_b200 import experts, i8, mx

from .test_mx import HALF, close, f64, numbers, step
from .test_mx_paths import counted  # noqa: F401  (sets the count of waits that have run out from the host, and back)

gpu = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def ends_of(counts, device="cuda"):
    return torch.tensor(np.cumsum(counts), dtype=torch.int32, device=device)


def clamped(ends, rows):
    """Each expert's rows as (first, last)."""
    out, at = [], 0
    for e in ends:
        end = max(at, min(int(e), rows))
        out.append((at, end))
        at = end
    return out


def formulas(x, w, spans, dy=None, bias=None):
    """y, dx, dw, db, and of the first three the sums of magnitudes."""
    rows, (E, n, k) = x.shape[0], w.shape
    y, ay = np.zeros((rows, n)), np.zeros((rows, n))
    out = {}
    for e, (a, b) in enumerate(spans):
        y[a:b], ay[a:b] = x[a:b] @ w[e].T, np.abs(x[a:b]) @ np.abs(w[e]).T
        if bias is not None:
            y[a:b] += bias[e]
    out["y"], out["ay"] = y, ay
    if dy is not None:
        dx, adx, dw, adw, db, adb = np.zeros((rows, k)), np.zeros((rows, k)), np.zeros(w.shape), np.zeros(w.shape), np.zeros((E, n)), np.zeros((E, n))
        for e, (a, b) in enumerate(spans):
            dx[a:b], adx[a:b] = dy[a:b] @ w[e], np.abs(dy[a:b]) @ np.abs(w[e])
            dw[e], adw[e] = dy[a:b].T @ x[a:b], np.abs(dy[a:b]).T @ np.abs(x[a:b])
            db[e], adb[e] = dy[a:b].sum(0), np.abs(dy[a:b]).sum(0)
        out |= {"dx": dx, "adx": adx, "dw": dw, "adw": adw, "db": db, "adb": adb}
    return out


def cut(length):
    return (length / 16 + 4) * 2 * HALF


def inputs(counts, behind, n, k, dtype, pad=0, seed=0):
    """x, w, dy, bias on the device; rows behind the last end are NaN, what is between rows too."""
    rows = sum(counts) + behind
    x, dy = numbers(seed + 1, rows, k, DT[dtype], pad), numbers(seed + 3, rows, n, DT[dtype], pad)
    wide = [torch.full((rows, t.shape[1] + pad), float("nan"), dtype=DT[dtype], device="cuda") for t in (x, dy)]
    for t, v in zip(wide, (x, dy)):
        t[:rows - behind, :v.shape[1]] = v[:rows - behind]
    w = numbers(seed + 2, len(counts) * n, k, DT[dtype]).reshape(len(counts), n, k).cuda()
    return wide[0][:, :k], w, wide[1][:, :n], numbers(seed + 4, len(counts), n, DT[dtype]).cuda()


def clean(t, behind):
    """As the formulas see it: what is behind the last end counts for nothing."""
    t = f64(t).copy()
    t[t.shape[0] - behind:] = 0
    return t


# ------------------------------------------------------------------------------------------------- without a GPU

def test_calls_without_a_context_are_refused():
    lib = gb.load_library()
    assert lib.galv_expert_matmul(None, 1, 1, 1, 1, None, None, 1, None, 1, None, None, 1, 1, None, 0, None) == gb.ERR_INVALID_ARG
    assert lib.galv_expert_input_grad(None, 1, 1, 1, 1, None, None, 1, None, 1, None, 1, 1, None, 0, None) == gb.ERR_INVALID_ARG
    assert lib.galv_expert_weight_grad(None, 1, 1, 1, 1, None, None, 1, None, 1, 1, None, None, 1, None, 0, None) == gb.ERR_INVALID_ARG
    assert lib.galv_expert_bias_grad(None, 1, 1, 1, None, None, 1, 1, None, 1, None) == gb.ERR_INVALID_ARG
    assert lib.galv_expert_backward(None, 1, 1, 1, 1, None, None, 1, None, 1, None, 1, 1, None, 1, None, None, None, 0, None) == gb.ERR_INVALID_ARG
    assert lib.galv_expert_matmul_workspace_bytes(None, 1, 1, 1, 1, None, 1, None, 1) == lib.galv_expert_weight_grad_workspace_bytes(None, 1, 1, 1, 1, None, 1, None, 1) == 0


def test_distance_of_moved_rows():
    lib = gb.load_library()
    for cols in [*range(1, 1400), 2 ** 20 + 1, 2 ** 31 - 129]:
        pitch = lib.galv_expert_pitch(cols)
        assert pitch % 8 == 0 and cols <= pitch < cols + 64
    assert lib.galv_expert_pitch(0) == lib.galv_expert_pitch(-5) == lib.galv_expert_pitch(2 ** 31 - 128) == 0


@pytest.mark.parametrize("need", [(1, 1, 1), (0, 1, 0), (1, 0, 1)])
@pytest.mark.parametrize("rows,n,k", [(6, 8, 64), (4096, 256, 256), (5, 3, 7)])
def test_gradients_get_the_workspace_that_the_library_asks_for(rows, n, k, need, monkeypatch):
    """A library that wants one for every weight gradient, and for whatever is off 16-byte boundaries: how it splits rows is its own affair."""
    given = []

    class Library:
        def galv_expert_matmul_workspace_bytes(self, *a):
            return 0

        def galv_expert_matmul(self, *a):
            pass

        def galv_expert_backward_workspace_bytes(self, rows, experts, n, k, dy, x, w):
            return 512 if x[0] or dy[1] % 8 or w[1] % 8 else 0

        def galv_expert_backward(self, *a):
            given.append(a)

    monkeypatch.setattr(experts, "_on", lambda *a: Library())
    leaves = [torch.zeros(s, dtype=torch.bfloat16).requires_grad_(bool(r)) for s, r in zip(((rows, k), (2, n, k), (2, n)), need)]
    experts.linear(leaves[0], leaves[1], torch.zeros(2, dtype=torch.int32), leaves[2]).sum().backward()
    (*_, dx, dw, db, ws), = given
    assert [dx[0] is not None, dw is not None, db is not None] == [bool(r) for r in need]
    assert (ws is not None and ws.numel() == 512) if need[1] or n % 8 or k % 8 else ws is None


B = torch.bfloat16
X, W, E3 = torch.zeros(6, 64, dtype=B), torch.zeros(3, 8, 64, dtype=B), torch.zeros(3, dtype=torch.int32)
W8 = i8.Packed(torch.zeros(24, 64, dtype=torch.int8), torch.zeros(24), 24, 64)
X8 = i8.Packed(torch.zeros(6, 64, dtype=torch.int8), torch.zeros(6), 6, 64)


@pytest.mark.parametrize("call", [
    lambda: experts.matmul(X, W, E3),                                              # not on a GPU
    lambda: experts.matmul(X.float(), W.float(), E3),                              # 32 bits
    lambda: experts.matmul(X, W.half(), E3),
    lambda: experts.matmul(X[:, :63], W, E3),
    lambda: experts.matmul(X[0], W, E3),
    lambda: experts.matmul(X, W[0], E3),
    lambda: experts.matmul(X, W, E3.long()),
    lambda: experts.matmul(X, W, E3[:2]),
    lambda: experts.matmul(X, W[:0], E3[:0]),
    lambda: experts.matmul(X, torch.zeros(1025, 8, 64, dtype=B), torch.zeros(1025, dtype=torch.int32)),
    lambda: experts.matmul(X, W, E3, torch.zeros(3, 8)),
    lambda: experts.matmul(X, W, E3, torch.zeros(8, dtype=B)),
    lambda: experts.matmul(X, W, E3, dtype=torch.float32),
    lambda: experts.matmul(X, W8, E3),
    lambda: experts.matmul(X, W8, E3[:, None]),
    lambda: experts.matmul(X, W8, torch.zeros(5, dtype=torch.int32)),              # 24 rows
    lambda: experts.matmul(X, W8, E3, torch.zeros(3, 8)),
    lambda: experts.matmul(X8, W, E3),
    lambda: experts.matmul(X8, W8, E3, dtype=torch.float64),
    lambda: experts.matmul(X8, W8, E3),
    lambda: experts.input_grad(torch.zeros(6, 9, dtype=B), W, E3),
    lambda: experts.input_grad(torch.zeros(6, 8, dtype=B), W, E3),
    lambda: experts.weight_grad(torch.zeros(6, 8, dtype=B), X, E3),
    lambda: experts.weight_grad(torch.zeros(5, 8, dtype=B), X, E3),
    lambda: experts.weight_grad(torch.zeros(6, 8, dtype=torch.float16), X, E3),
    lambda: experts.weight_grad(torch.zeros(6, 8, dtype=B), X, E3, torch.float16),
    lambda: experts.weight_grad(torch.zeros(6, 8, dtype=B), X, E3, base=torch.zeros(3, 8, 63, dtype=B)),
    lambda: experts.weight_grad(torch.zeros(6, 8, dtype=B), X, E3, out=torch.zeros(3, 64, 8, dtype=B).transpose(1, 2)),
    lambda: experts.bias_grad(torch.zeros(6, 8, dtype=B), E3),
    lambda: experts.bias_grad(torch.zeros(6, 8, dtype=B), E3, torch.float16),
    lambda: experts.linear(X, W, E3),
    lambda: experts.linear(X, W, E3.long()),
])
def test_refusals(call):
    with pytest.raises(ValueError):
        call()


# ------------------------------------------------------------------------------------------------- forward and gradients

CASES = [([1], 0, 1, 1), ([1], 0, 16, 2048), ([2, 0, 1], 1, 100, 64), ([0, 0, 5, 0], 0, 33, 70), ([31, 32, 33], 2, 257, 129), ([256], 0, 256, 256), ([300, 0, 257, 1], 70, 300, 200),
         ([1100, 40], 0, 130, 96), ([3] * 40, 5, 65, 130), ([0] * 7, 9, 40, 24), ([17, 200, 600, 2, 0, 64], 3, 513, 320), ([2500], 100, 24, 40), ([1100, 0, 6000], 5, 300, 77), ([9000], 0, 70, 264), ([100, 6300, 5], 33, 128, 130)]


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("counts,behind,n,k", CASES)
def test_forward_and_gradients(counts, behind, n, k, dtype):
    for pad in (0, 3, 8):
        x, w, dy, bias = inputs(counts, behind, n, k, dtype, pad)
        ends, spans = ends_of(counts), clamped(np.cumsum(counts), x.shape[0])
        f = formulas(clean(x, behind), f64(w), spans, clean(dy, behind), f64(bias))
        dt = DT[dtype]
        close(experts.matmul(x, w, ends, bias), f["y"], cut(k) * f["ay"] + HALF * np.abs(f["y"]) + step(dt, f["y"]), "y")
        close(experts.input_grad(dy, w, ends), f["dx"], cut(n) * f["adx"] + step(dt, f["dx"]), "dx")
        most = max(counts)
        for out in (dt, torch.float32):
            tol = (cut(min(most, 768)) + most / 768 * HALF) * f["adw"] + step(out, f["dw"])
            close(experts.weight_grad(dy, x, ends, out), f["dw"], tol, "dw")
            base = numbers(5, len(counts) * n, k, out).reshape(len(counts), n, k).cuda()
            total = f["dw"] + f64(base)
            onto = experts.weight_grad(dy, x, ends, base=base)
            close(onto, total, tol + step(out, total) + HALF * np.abs(total), "dw onto base")
            assert experts.weight_grad(dy, x, ends, base=base, out=base) is base and torch.equal(base, onto)
            tol = (most / 64 + 16) * HALF * f["adb"] + step(out, f["db"])
            close(experts.bias_grad(dy, ends, out), f["db"], tol, "db")


@gpu
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("counts,behind,n,k", CASES + [([1, 0, 2, 0, 0, 1], 0, 2100, 4096), ([9, 55], 0, 300, 1000)])
def test_products_in_8_bit_integers(counts, behind, n, k, dtype):
    rows = sum(counts) + behind
    dt = DT[dtype]
    x = numbers(1, rows, k, dt).cuda()
    x[rows - behind:] = float("nan")
    w = i8.pack(numbers(2, len(counts) * n, k, torch.float32).cuda())
    bias = numbers(3, len(counts), n, dt).cuda()
    p = i8.pack(x)
    ends, spans = ends_of(counts), clamped(np.cumsum(counts), rows)
    sx = np.where(np.isnan(f64(p.scales)), 0, f64(p.scales))
    a, b = p.codes.cpu().numpy()[:, :k].astype(np.float64), w.codes.cpu().numpy()[:, :k].astype(np.float64).reshape(len(counts), n, k)
    want, size = np.zeros((rows, n)), np.zeros((rows, n))
    for e, (s, t) in enumerate(spans):
        v = (a[s:t] @ b[e].T) * sx[s:t, None] * f64(w.scales).reshape(-1, n)[e]
        want[s:t], size[s:t] = v + f64(bias)[e], np.abs(v)
    got = experts.matmul(p, w, ends, bias, dt)
    close(got, want, 3 * HALF * size + 2 * HALF * np.abs(want) + step(dt, want))
    assert torch.equal(experts.matmul(x, w, ends, bias), got)


@gpu
@pytest.mark.parametrize("counts,behind,n,k", [([300], 0, 20, 8192), ([70, 0, 130], 9, 136, 4099), ([64, 64, 1], 0, 33, 2048), ([100], 3, 4096, 20), ([65], 0, 9000, 24)])
def test_long_sums_for_few_results(counts, behind, n, k):
    """More than 64 rows, whose tiles of 64 clusters take: forward along the weights' rows, the input gradient across them, and the same rows in 8-bit integers."""
    x, w, dy, bias = inputs(counts, behind, n, k, "bf16")
    ends, spans = ends_of(counts), clamped(np.cumsum(counts), x.shape[0])
    f = formulas(clean(x, behind), f64(w), spans, clean(dy, behind), f64(bias))
    close(experts.matmul(x, w, ends, bias), f["y"], cut(k) * f["ay"] + HALF * np.abs(f["y"]) + step(B, f["y"]), "y")
    close(experts.input_grad(dy, w, ends), f["dx"], cut(n) * f["adx"] + step(B, f["dx"]), "dx")
    p, q = i8.pack(x), i8.pack(w.view(-1, k))
    got = experts.matmul(p, q, ends, dtype=torch.float32)
    a, b = p.codes[:, :k].double(), q.codes[:, :k].double().view(len(counts), n, k)
    want = torch.zeros_like(got, dtype=torch.float64)
    for e, (s, t) in enumerate(spans):
        want[s:t] = (a[s:t] @ b[e].t()) * p.scales[s:t, None].double() * q.scales.view(-1, n)[e].double()
    assert ((got.double() - want).abs() <= 4 * HALF * want.abs()).all()
    assert torch.equal(experts.matmul(x.float(), q, ends), got)


@gpu
def test_ends_that_fall_or_leave_the_rows():
    rows, n, k = 100, 70, 64
    x, dy = numbers(1, rows, k, B).cuda(), numbers(3, rows, n, B).cuda()
    for ends in ([50, 20, 120, 60], [-5, 40, 30, 2 ** 31 - 1], [-2 ** 31, -1, 0, 10], [100, 100, 0, 100], [200, 0, 0, 0]):
        w = numbers(2, 4 * n, k, B).reshape(4, n, k).cuda()
        spans = clamped(ends, rows)
        f = formulas(f64(x), f64(w), spans, f64(dy))
        e = torch.tensor(ends, dtype=torch.int32, device="cuda")
        close(experts.matmul(x, w, e), f["y"], cut(k) * f["ay"] + step(B, f["y"]))
        close(experts.input_grad(dy, w, e), f["dx"], cut(n) * f["adx"] + step(B, f["dx"]))
        close(experts.weight_grad(dy, x, e), f["dw"], cut(rows) * f["adw"] + step(B, f["dw"]))
        close(experts.bias_grad(dy, e), f["db"], 20 * HALF * f["adb"] + step(B, f["db"]))
        assert torch.equal(experts.matmul(x, i8.pack(w.view(-1, k)), e), experts.matmul(x, i8.pack(w.view(-1, k)), torch.tensor([b for _, b in spans], dtype=torch.int32, device="cuda")))


@gpu
def test_what_is_no_number_stays_with_its_expert():
    counts = [5, 300, 70, 1, 20]
    x, w, dy, bias = inputs(counts, 4, 300, 200, "bf16")
    ends = ends_of(counts)

    def all_of():
        return experts.matmul(x, w, ends), experts.input_grad(dy, w, ends), experts.weight_grad(dy, x, ends, torch.float32), experts.bias_grad(dy, ends)
    before = all_of()
    x[310], dy[311, 5], w[3, 0, 0] = float("inf"), float("nan"), float("nan")      # rows 305 .. 374 are the third expert's
    after = all_of()
    assert not torch.isfinite(after[0][310]).any() and torch.isnan(after[1][311]).all() and torch.isnan(after[2][2, 5]).all() and torch.isnan(after[3][2, 5])
    rows = [r for r in range(len(x)) if r not in (310, 311, 375)]
    assert all(torch.equal(a[rows], b[rows]) for a, b in zip(before[:2], after[:2]))
    others = [0, 1, 3, 4]
    assert torch.equal(before[2][others], after[2][others]) and torch.equal(before[3][others], after[3][others])


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("out", ["same", "f32"])
def test_weight_gradients_onto_earlier_ones(dtype, out):
    counts, n, k = [40, 0, 1300, 3], 300, 131
    x, w, dy, _ = inputs(counts, 6, n, k, dtype)
    to = DT[dtype] if out == "same" else torch.float32
    base = numbers(9, 4 * n, k, to).reshape(4, n, k).cuda()
    f = formulas(clean(x, 6), f64(w), clamped(np.cumsum(counts), len(x)), clean(dy, 6))
    want = f["dw"] + f64(base)
    tol = (cut(768) + 3 * HALF) * f["adw"] + HALF * np.abs(want) + step(to, want)
    ends = ends_of(counts)
    fresh = experts.weight_grad(dy, x, ends, base=base)
    assert fresh.dtype == to
    close(fresh, want, tol)
    assert torch.equal(fresh[1], base[1])                                          # no rows
    assert experts.weight_grad(dy, x, ends, base=base, out=base) is base and torch.equal(base, fresh)


@gpu
@pytest.mark.parametrize("n, k", [(1, 1), (3, 5), (33, 7), (40, 31), (35, 33), (7, 127), (130, 129), (257, 134), (65, 300), (290, 385)])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_weight_gradients_whose_rows_start_anywhere(n, k, out):
    """Results at every distance from a 16-byte boundary, with a base at another one: whole numbers, whose sums stay below 256 and are exact, and nothing beside them is written."""
    counts, E, to = [5, 0, 20, 1], 4, DT[out]
    rng = np.random.default_rng(n * 1000 + k)
    x, dy = (torch.tensor(rng.integers(-2, 3, (sum(counts), c)), dtype=torch.bfloat16).cuda() for c in (k, n))
    base = torch.tensor(rng.integers(-100, 101, (E, n, k)), dtype=to).cuda()
    ends, size = ends_of(counts), E * n * k
    dw = torch.tensor(formulas(f64(x), np.zeros((E, n, k)), clamped(np.cumsum(counts), len(x)), f64(dy))["dw"], dtype=to).cuda()
    for at in range(0, 16 // to.itemsize, 1 if k == 129 else 3):
        for beside in (None, 0, 1):
            around = torch.full((size + 64,), 77., dtype=to, device="cuda")
            result = around[at:at + size].view(E, n, k)
            if beside is None:
                first = None
            elif beside == 0:
                first = result.copy_(base)
            else:
                first = torch.zeros(size + 64, dtype=to, device="cuda")[at + beside:at + beside + size].view(E, n, k).copy_(base)
            experts.weight_grad(dy, x, ends, to, base=first, out=result)
            assert torch.equal(result, dw if first is None else dw + base), (at, beside)
            assert (around[:at] == 77).all() and (around[at + size:] == 77).all()


@gpu
@pytest.mark.parametrize("rows", [0, 3])
def test_nobody_has_rows(rows):
    x, dy, w = torch.full((rows, 40), float("nan"), dtype=B, device="cuda"), torch.full((rows, 24), float("nan"), dtype=B, device="cuda"), torch.ones(5, 24, 40, dtype=B, device="cuda")
    ends = torch.zeros(5, dtype=torch.int32, device="cuda")
    assert not experts.matmul(x, w, ends, torch.ones(5, 24, dtype=B, device="cuda")).any() and experts.matmul(x, w, ends).shape == (rows, 24)
    assert not experts.matmul(x, i8.pack(w.view(-1, 40)), ends).any()
    assert not experts.input_grad(dy, w, ends).any() and not experts.weight_grad(dy, x, ends).any() and not experts.bias_grad(dy, ends).any()
    base = numbers(1, 120, 40, torch.float32).view(5, 24, 40).cuda()
    assert torch.equal(experts.weight_grad(dy, x, ends, base=base), base)
    leaves = [t.clone().requires_grad_() for t in (x, w, torch.ones(5, 24, dtype=B, device="cuda"))]
    y = experts.linear(leaves[0], leaves[1], ends, leaves[2])
    grads = torch.autograd.grad(y, leaves, dy)
    assert not y.any() and all(g.shape == t.shape and not g.any() for g, t in zip(grads, leaves))


@gpu
def test_one_expert_without_ends():
    """The library's calls take no ends where one expert has all rows: plain products and gradients."""
    rows, n, k = 300, 136, 72
    x, w, dy, bias = inputs([rows], 0, n, k, "bf16")
    ends = ends_of([rows])
    want = experts.matmul(x, w, ends, bias), experts.input_grad(dy, w, ends), experts.weight_grad(dy, x, ends), experts.bias_grad(dy, ends)
    y, dx, dw, db = (torch.full_like(t, float("nan")) for t in want)
    g = mx.context(0)
    g.galv_expert_matmul(rows, 1, n, k, None, (x.data_ptr(), k), (w.data_ptr(), k), bias, (y.data_ptr(), n), gb.BF16, None)
    g.galv_expert_backward(rows, 1, n, k, None, (dy.data_ptr(), n), (x.data_ptr(), k), (w.data_ptr(), k), gb.BF16, (dx.data_ptr(), k), dw, db, None)
    assert all(torch.equal(a, b) for a, b in zip((y, dx, dw, db), want))
    with pytest.raises(gb.GalvError):
        g.galv_expert_matmul(rows, 2, n // 2, k, None, (x.data_ptr(), k), (w.data_ptr(), k), None, (y.data_ptr(), n // 2), gb.BF16, None)


@gpu
def test_refusals_of_the_library():
    """Nothing is launched for pointers, strides, sizes and workspaces that cannot be."""
    g = mx.context(0)
    x, w = torch.zeros(8, 64, dtype=B, device="cuda"), torch.zeros(2, 16, 64, dtype=B, device="cuda")
    ends, y, ws = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(8, 16, dtype=B, device="cuda"), torch.zeros(4096, dtype=torch.uint8, device="cuda")
    xp, wp, yp = x.data_ptr(), w.data_ptr(), y.data_ptr()
    calls = [((8, 2, 16, 64, ends, (xp, 64), (wp, 64), None, (yp, 15), gb.BF16, None), gb.ERR_INVALID_ARG),       # rows of y overlap
             ((8, 2, 16, 64, ends, (xp, 63), (wp, 64), None, (yp, 16), gb.BF16, None), gb.ERR_INVALID_ARG),
             ((8, 2, 16, 64, ends, (xp, 64), (wp, 63), None, (yp, 16), gb.BF16, None), gb.ERR_INVALID_ARG),
             ((8, 2, 16, 64, ends, (xp + 1, 64), (wp, 64), None, (yp, 16), gb.BF16, None), gb.ERR_INVALID_ARG),
             ((8, 2, 16, 64, ends, (None, 64), (wp, 64), None, (yp, 16), gb.BF16, None), gb.ERR_INVALID_ARG),
             ((8, 2, 16, 64, ends, (xp, 64), (wp, 64), None, (yp, 16), gb.F32, None), gb.ERR_INVALID_ARG),
             ((8, 1025, 16, 64, ends, (xp, 64), (wp, 64), None, (yp, 16), gb.BF16, None), gb.ERR_INVALID_ARG),
             ((8, 0, 16, 64, ends, (xp, 64), (wp, 64), None, (yp, 16), gb.BF16, None), gb.ERR_INVALID_ARG),
             ((8, 2, 0, 64, ends, (xp, 64), (wp, 64), None, (yp, 16), gb.BF16, None), gb.ERR_INVALID_ARG),
             ((-1, 2, 16, 64, ends, (xp, 64), (wp, 64), None, (yp, 16), gb.BF16, None), gb.ERR_INVALID_ARG),
             ((2 ** 31, 2, 16, 64, ends, (xp, 64), (wp, 64), None, (yp, 16), gb.BF16, None), gb.ERR_INVALID_ARG),
             ((4, 2, 16, 63, ends, (xp, 65), (wp, 63), None, (yp, 16), gb.BF16, None), gb.ERR_WORKSPACE),          # rows to be moved
             ((4, 2, 16, 63, ends, (xp, 65), (wp, 63), None, (yp, 16), gb.BF16, ws[:256]), gb.ERR_WORKSPACE),
             ((4, 2, 16, 63, ends, (xp, 65), (wp, 63), None, (yp, 16), gb.BF16, ws[1:]), gb.ERR_WORKSPACE)]
    for args, code in calls:
        with pytest.raises(gb.GalvError) as e:
            g.galv_expert_matmul(*args)
        assert e.value.code == code
    q = i8.pack(x)
    s = q.scales
    for args in ((8, 2, 16, 131072, ends, q.codes, s, q.codes, s, None, (yp, 16), gb.BF16), (8, 2, 16, 64, None, q.codes, s, q.codes, s, None, (yp, 16), gb.BF16),
                 (8, 2, 16, 64, ends, q.codes[:, 1:], s, q.codes, s, None, (yp, 16), gb.BF16), (8, 2, 16, 64, ends, q.codes, s, q.codes, s, None, (yp, 16), 8)):
        with pytest.raises(gb.GalvError) as e:
            g.galv_i8_matmul(*args)
        assert e.value.code == gb.ERR_INVALID_ARG
    with pytest.raises(gb.GalvError) as e:
        g.galv_i8_linear(8, 2, 16, 64, ends, (xp, 64), q.codes, s, None, (yp, 16), gb.BF16, None)
    assert e.value.code == gb.ERR_WORKSPACE
    assert not y.any()


@gpu
def test_products_raise_behind_a_wait_that_ran_out(counted):                        # noqa: F811
    """The count is the library's own: an earlier product's void result is said by the next call of any of them, once."""
    x, w, dy, _ = inputs([30, 70], 0, 40, 64, "bf16")
    ends, p, q = ends_of([30, 70]), i8.pack(x), i8.pack(w.view(-1, 64))
    calls = [lambda: experts.matmul(x, w, ends), lambda: experts.input_grad(dy, w, ends), lambda: experts.weight_grad(dy, x, ends), lambda: experts.matmul(p, q, ends),
             lambda: experts.matmul(x, q, ends), lambda: i8.matmul(p, q), lambda: i8.linear(x, q)]
    want = [c() for c in calls]
    for c, right in zip(calls, want):
        counted(1)
        with pytest.raises(gb.GalvError) as e:
            c()
        assert e.value.code == gb.ERR_TIMEOUT
        assert torch.equal(c(), right)


@gpu
def test_offsets_past_32_bits():
    """Results, inputs, weights and gradients of more than 2^31 elements: rows and experts on both sides of it."""
    n, k = 32768, 64
    rows = 2 ** 31 // n + 300
    counts = [rows - 270, 0, 250]
    g = torch.Generator(device="cuda").manual_seed(1)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.float16)
    x, w, ends = make(rows, k), make(3, n, k), ends_of(counts)
    y = experts.matmul(x, w, ends)
    for a, b, e in ((0, 40, 0), (rows - 310, rows - 270, 0), (rows - 270, rows - 20, 2)):
        want = x[a:b].double() @ w[e].double().t()
        size = x[a:b].double().abs() @ w[e].double().abs().t()
        assert ((y[a:b].double() - want).abs() <= cut(k) * size + want.abs() * 2 ** -11 + 2.0 ** -25).all()
    assert not y[rows - 20:].any()
    dx = experts.input_grad(y, w, ends)                                              # y in the place of a gradient
    a, b = rows - 270, rows - 250
    want, size = y[a:b].double() @ w[2].double(), y[a:b].double().abs() @ w[2].double().abs()
    ok = (dx[a:b].double() - want).abs() <= cut(n) * size + want.abs() * 2 ** -11 + 2.0 ** -25
    assert (ok | (want.abs() > 65000)).all() and not dx[rows - 20:].any()
    db = experts.bias_grad(y, ends, torch.float32)
    want, size = y[a:rows - 20].double().sum(0), y[a:rows - 20].double().abs().sum(0)
    assert ((db[2].double() - want).abs() <= 24 * HALF * size).all()
    del y, dx
    E, n, k = 33, 8192, 8192                                                         # 2.2e9 weights
    counts = [5] * E
    x, dy, w, ends = make(5 * E, k), make(5 * E, n), make(E, n, k), ends_of(counts)
    y, dx, dw = experts.matmul(x, w, ends), experts.input_grad(dy, w, ends), experts.weight_grad(dy, x, ends)
    for e in (0, E - 1):
        at = slice(5 * e, 5 * e + 5)
        for got, u, v in ((y[at], x[at], w[e].t()), (dx[at], dy[at], w[e]), (dw[e], dy[at].t(), x[at])):
            want, size = u.double() @ v.double(), u.double().abs() @ v.double().abs()
            assert ((got.double() - want).abs() <= cut(u.shape[1]) * size + want.abs() * 2 ** -11 + 2.0 ** -25).all()
    p = i8.pack(w.view(-1, k))
    few = i8.Packed(p.codes[(E - 1) * n:], p.scales[(E - 1) * n:], n, k)
    assert torch.equal(experts.matmul(x, p, ends)[-5:], i8.linear(x[-5:], few))


@gpu
def test_many_experts():
    """1024 of them, most without rows."""
    g = np.random.default_rng(5)
    counts = (g.integers(0, 6, 1024) * (g.random(1024) < 0.2)).tolist()
    x, w, dy, bias = inputs(counts, 1, 40, 48, "bf16")
    ends = ends_of(counts)
    f = formulas(clean(x, 1), f64(w), clamped(np.cumsum(counts), len(x)), clean(dy, 1), f64(bias))
    close(experts.matmul(x, w, ends, bias), f["y"], cut(48) * f["ay"] + HALF * np.abs(f["y"]) + step(B, f["y"]))
    close(experts.input_grad(dy, w, ends), f["dx"], cut(40) * f["adx"] + step(B, f["dx"]))
    close(experts.weight_grad(dy, x, ends), f["dw"], cut(8) * f["adw"] + step(B, f["dw"]))
    close(experts.bias_grad(dy, ends), f["db"], 24 * HALF * f["adb"] + step(B, f["db"]))


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_strides_and_views(dtype):
    """Transposed, expanded, negative and shifted operands give what contiguous copies give."""
    counts, n, k = [40, 3, 90], 72, 80
    x, w, dy, bias = inputs(counts, 0, n, k, dtype)
    ends = ends_of(counts)
    want = experts.matmul(x, w, ends, bias), experts.input_grad(dy, w, ends), experts.weight_grad(dy, x, ends), experts.bias_grad(dy, ends)
    shifted = torch.empty(w.numel() + 1, dtype=w.dtype, device="cuda")[1:].view_as(w).copy_(w)
    odd = torch.empty(len(x), k + 1, dtype=x.dtype, device="cuda")[:, 1:].copy_(x)
    for xv, wv, dv in ((x.t().contiguous().t(), w.transpose(1, 2).contiguous().transpose(1, 2), dy.t().contiguous().t()),
                       (torch._neg_view(-x), torch._neg_view(-w), torch._neg_view(-dy)), (odd, shifted, dy)):
        got = experts.matmul(xv, wv, ends, bias), experts.input_grad(dv, wv, ends), experts.weight_grad(dv, xv, ends), experts.bias_grad(dv, ends)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    one = dy[:1].expand(len(x), n)
    assert torch.equal(experts.bias_grad(one, ends), experts.bias_grad(one.contiguous(), ends)) and torch.equal(experts.weight_grad(one, x, ends), experts.weight_grad(one.contiguous(), x, ends))
    padded = torch.full((3, n, k + 8), float("nan"), dtype=w.dtype, device="cuda")[:, :, :k].copy_(w)      # rows further apart than they are long
    assert torch.equal(experts.matmul(x, padded, ends, bias), want[0]) and torch.equal(experts.input_grad(dy, padded, ends), want[1])
    strided = torch.zeros(6, dtype=torch.int32, device="cuda")
    strided[::2] = ends
    assert torch.equal(experts.matmul(x, w, strided[::2], bias), want[0])


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("k", [7, 100, 511, 513, 1365])
@pytest.mark.parametrize("odd", ["both", "x", "w"])
def test_what_the_forward_product_has_moved_lies_where_the_header_says(k, odd, dtype):
    """Of operands off 16-byte boundaries: read back by the header's rule, and handed on to the three gradients in one call."""
    g, counts, n = mx.context(0), [60, 0, 17], 40
    rows, E, number = sum(counts), len(counts), gb._DTYPES[DT[dtype]]
    x, w, dy, _ = inputs(counts, 0, n, k, dtype)
    ends, wide = ends_of(counts), (k + 7) // 8 * 8
    apart = lambda t: torch.zeros(*t.shape[:-1], wide, dtype=t.dtype, device="cuda")[..., :k].copy_(t)      # rows that bulk copies take as they are
    xv, wv = x if odd != "w" else apart(x), w if odd != "x" else apart(w)
    xm, wm = gb._matrix(xv), gb._matrices(wv)
    ws = torch.full((g.galv_expert_matmul_workspace_bytes(rows, E, n, k, xm, wm),), 255, dtype=torch.uint8, device="cuda")
    y = torch.empty(rows, n, dtype=x.dtype, device="cuda")
    g.galv_expert_matmul(rows, E, n, k, ends, xm, wm, None, (y.data_ptr(), n), number, ws)
    pitch, at = g.galv_expert_pitch(k), 0
    assert pitch >= k and pitch % 8 == 0
    back = []
    for t, view, moved in ((x, xv, odd != "w"), (w, wv, odd != "x")):
        count = t.numel() // k
        if moved:
            held = ws[at:at + count * pitch * 2].view(x.dtype).view(*t.shape[:-1], pitch)
            assert torch.equal(held[..., :k], t) and not held[..., k:].any()
            at += (count * pitch * 2 + 255) & ~255
            back.append(held[..., :k])
        else:
            back.append(view)
    assert at == ws.numel()
    operands = gb._matrix(dy), gb._matrix(back[0]), gb._matrices(back[1])
    size = g.galv_expert_backward_workspace_bytes(rows, E, n, k, *operands)
    assert size == 0                                                                 # nothing is moved again
    dx, dw, db = torch.empty(rows, k, dtype=x.dtype, device="cuda"), torch.empty(E, n, k, dtype=x.dtype, device="cuda"), torch.empty(E, n, dtype=x.dtype, device="cuda")
    g.galv_expert_backward(rows, E, n, k, ends, *operands, number, (dx.data_ptr(), k), dw, db, None)
    assert torch.equal(y, experts.matmul(x, w, ends)) and torch.equal(dx, experts.input_grad(dy, w, ends))
    assert torch.equal(dw, experts.weight_grad(dy, x, ends)) and torch.equal(db, experts.bias_grad(dy, ends))
    kept = experts._moved(xv, wv, ws)                                                # what the differentiable function keeps
    assert torch.equal(kept[0], x) and torch.equal(kept[1], w) and [t.data_ptr() for t in kept] == [t.data_ptr() for t in back]


@gpu
def test_what_lies_right_is_not_moved():
    """The rule that saves asking the library, against what it says: operands of all starts, distances and sizes."""
    g, lie = mx.context(0), experts._lie
    for n, k in ((1, 1), (8, 8), (40, 7), (33, 64), (1365, 2731), (4096, 4096)):
        for at in (0, 2, 8, 16, 256):
            for pad in (0, 1, 4, 8, 24, 1 << 39):
                for rows, e in ((100, 1), (100, 5), (50000, 1), (50000, 5)):      # more are split in parts
                    x, w, dy = (4096 + at, k + pad), (8192 + at // 2 * 2, k + pad), (1 << 20, n + pad)
                    sizes = rows, e, n, k
                    if lie(n, x, w):
                        assert g.galv_expert_matmul_workspace_bytes(*sizes, x, w) == 0
                    else:                                                            # the rows' limit is taken for the matrices' too
                        assert g.galv_expert_matmul_workspace_bytes(*sizes, x, w) > 0 or n * (k + pad) >= 1 << 39
                    if lie(n, dy, w):
                        assert g.galv_expert_backward_workspace_bytes(*sizes, dy, (None, 0), w) == 0
                    if lie(n, dy, x):
                        assert g.galv_expert_backward_workspace_bytes(*sizes, dy, x, (None, 0)) == g.galv_expert_backward_workspace_bytes(*sizes, (1 << 20, 4096), (1 << 21, 4096), (None, 0))


# ------------------------------------------------------------------------------------------------- as a differentiable function

@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_gradients_are_those_of_the_function(dtype):
    """Small whole numbers, with which nothing rounds: the function's differences along any direction are what its gradients say."""
    g = torch.Generator().manual_seed(1)
    counts, n, k = [4, 0, 33, 7], 24, 18
    dt, rows = DT[dtype], 46
    draw = lambda *s: torch.randint(-1, 2, s, generator=g).to(dt).cuda()
    x, w, b, dy = draw(rows, k), draw(4, n, k), draw(4, n), draw(rows, n)
    ends = ends_of(counts)
    for t in (x, w, b):
        t.requires_grad_()
    y = experts.linear(x, w, ends, b)
    dx, dw, db = torch.autograd.grad(y, (x, w, b), dy)
    along = [draw(*t.shape) for t in (x, w, b)]
    loss = lambda x, w, b: (experts.linear(x, w, ends, b).double() * dy.double()).sum()
    with torch.no_grad():
        for i, grad in enumerate((dx, dw, db)):
            args = [x, w, b]
            args[i] = args[i] + along[i]
            assert loss(*args) - loss(x, w, b) == (grad.double() * along[i].double()).sum()
    assert not y[44:].any() and not dx[44:].any()


@gpu
@pytest.mark.parametrize("n,k,pad", [(24, 40, 0), (33, 41, 0), (33, 41, 7), (24, 40, 3), (24, 45, 3), (1, 1, 0)])
def test_linear_takes_only_the_gradients_that_are_asked_for(n, k, pad):
    counts = [10, 0, 30]
    x, w, dy, b = inputs(counts, 2, n, k, "bf16", pad)
    x = x.nan_to_num(0.0)
    ends = ends_of(counts)
    want = experts.matmul(x, w, ends, b), experts.input_grad(dy, w, ends), experts.weight_grad(dy, x, ends), experts.bias_grad(dy, ends)
    for need in ((1, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1)):
        leaves = [t.detach().clone().requires_grad_(bool(r)) for t, r in zip((x, w, b), need)]
        y = experts.linear(leaves[0], leaves[1], ends, leaves[2])
        assert torch.equal(y, want[0])
        y.backward(dy)
        assert all((t.grad is None) if not r else torch.equal(t.grad, g) for t, r, g in zip(leaves, need, want[1:]))
    with torch.autocast("cuda", dtype=torch.float16):
        assert torch.equal(experts.linear(x, w, ends, b), want[0])
    with torch.no_grad():
        assert not experts.linear(x.requires_grad_(), w, ends).requires_grad


@gpu
def test_captured_with_other_ends():
    """A training step's products in a graph: new inputs and new ends at each replay, without anything that waits for them."""
    n, k, rows = 200, 136, 500
    sets = []
    for counts in ([100, 0, 300, 60], [0, 0, 0, 500], [1, 2, 3, 4]):
        behind = rows - sum(counts)
        x, w, dy, b = inputs(counts, behind, n, k, "bf16", seed=len(sets) * 10)
        sets.append((x.nan_to_num(3.0), w, dy.nan_to_num(5.0), b, ends_of(counts)))
    static = [t.clone() for t in sets[0]]

    def run():
        x, w, dy, b, ends = static
        y = experts.linear(x, w, ends, b)
        return (y.detach(), *torch.autograd.grad(y, (x, w, b), dy))
    for t in (static[0], static[1], static[3]):
        t.requires_grad_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    want = []
    for x, w, dy, b, ends in sets:
        want.append((experts.matmul(x, w, ends, b), experts.input_grad(dy, w, ends), experts.weight_grad(dy, x, ends), experts.bias_grad(dy, ends)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for i in (0, 1, 2, 1, 0):
        with torch.no_grad():
            for t, v in zip(static, sets[i]):
                t.copy_(v)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, want[i]))
    mx.check(0)


@gpu
@pytest.mark.parametrize("n", [1280, 1152, 1040])
def test_tiles_whose_sums_are_short(n):
    """One chunk a tile and ten tiles a pair of CTAs: each accumulator is summed into again as soon as both have moved it out.  n leaves the second of a pair all of the last tile's
    columns or none, and the first all or 16.  Whole numbers, with which nothing rounds."""
    g = torch.Generator(device="cuda").manual_seed(n)
    counts, rows = [20011, 0, 17, 19001], 39100
    ends = ends_of(counts)
    spans = clamped(ends, rows)
    draw = lambda most, *s: torch.randint(-most, most + 1, s, generator=g, device="cuda")
    plain = lambda u, v: torch.cat([u[a:b].float() @ v[e].float() for e, (a, b) in enumerate(spans)] + [torch.zeros(rows - spans[-1][1], v.shape[2], device="cuda")])
    x, w = draw(1, rows, 64).to(B), draw(1, 4, n, 64).to(B)
    qx, qw = draw(127, rows, 64).to(torch.int8), draw(127, 4, n, 64).to(torch.int8)
    px, pw = i8.Packed(qx, torch.ones(rows, device="cuda"), rows, 64), i8.Packed(qw, torch.ones(4 * n, device="cuda"), 4 * n, 64)
    dy, wt = draw(1, rows, 64).to(B), draw(1, 4, 64, n).to(B)
    want = plain(x, w.transpose(1, 2)), plain(qx, qw.transpose(1, 2)), plain(dy, wt)
    for _ in range(10):
        got = experts.matmul(x, w, ends), experts.matmul(px, pw, ends, dtype=torch.float32), experts.input_grad(dy, wt, ends)
        assert all(torch.equal(a.float(), b) for a, b in zip(got, want))


@gpu
def test_one_behind_the_other_eager_and_captured():
    """Kernels may begin before the one in front of them is over: each result is the next call's input or weights, fills and copies and other streams' work lie between, and a second
    replay finds what the first has left."""
    g = torch.Generator(device="cuda").manual_seed(9)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=B) / 8
    rows, d = 40, 512
    x0, w = make(rows, d), make(4, d, d)
    ends = ends_of([10, 0, 25, 5])
    side = torch.cuda.Stream()

    def chain(x):
        h = experts.matmul(x, w, ends)                                              # few rows
        p = i8.pack(h)
        h = i8.matmul(p, i8.pack(w[0])) + experts.matmul(h, i8.pack(w.view(-1, d)), ends)
        fork = torch.cuda.Event()
        fork.record()
        side.wait_event(fork)
        with torch.cuda.stream(side):
            other = experts.matmul(h, w, ends)
            done = torch.cuda.Event()
            done.record()
        torch.cuda.current_stream().wait_event(done)
        z = torch.zeros(3 * rows, d, dtype=B, device="cuda")
        z[:rows].copy_(other)
        z[rows:2 * rows] = h
        y = experts.matmul(z, w, ends_of_many)                                      # more than 64
        v = (y[:64].t() @ y[:64]).contiguous()                                      # weights that the next call reads at once
        q = i8.pack(v / 8)
        return i8.linear(y, q), i8.linear(y[:5], q), experts.weight_grad(y, z, ends_of_many)

    ends_of_many = ends_of([30, 50, 0, 37])
    want = chain(x0)
    torch.cuda.synchronize()
    for _ in range(20):
        assert all(torch.equal(a, b) for a, b in zip(chain(x0), want))
    x1 = make(rows, d)
    want1 = chain(x1)
    static = x0.clone()
    warm = torch.cuda.Stream()
    warm.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(warm):
        chain(static)
    torch.cuda.current_stream().wait_stream(warm)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = chain(static)
    for x, right in ((x1, want1), (x0, want), (x0, want), (x1, want1)):
        static.copy_(x)
        graph.replay()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, right))


@gpu
def test_two_streams_at_once():
    counts = [300, 20, 700]
    sets = [inputs(counts, 0, 264, 328, "f16", seed=s) for s in (0, 50)]
    ends = ends_of(counts)

    def run(x, w, dy, b):
        return experts.matmul(x, w, ends, b), experts.input_grad(dy, w, ends), experts.weight_grad(dy, x, ends), experts.matmul(x, i8.pack(w.view(-1, 328)), ends)
    want = [run(*s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[], []]
    for _ in range(10):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(run(*sets[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for i in (0, 1) for one in got[i] for a, b in zip(one, want[i]))


# ------------------------------------------------------------------------------------------------- as they are used together

def _route(scores, most):
    """Each token's `most` experts: (which row of which token, ends, weights of the rows), rows sorted by expert."""
    p = torch.softmax(scores.float(), 1)
    top, expert = p.topk(most, 1)
    order = torch.argsort(expert.flatten(), stable=True)
    ends = torch.bincount(expert.flatten(), minlength=scores.shape[1]).cumsum(0, dtype=torch.int32)
    return order // most, ends, top.flatten()[order], order


def _block(x, scores, w1, w2, b1):
    token, ends, weight, _ = _route(scores, 2)
    h = mx.activation(experts.linear(x[token], w1, ends, b1), "silu")
    out = experts.linear(h, w2, ends).float() * weight[:, None]
    return torch.zeros(x.shape, device=x.device).index_add_(0, token, out)


@gpu
def test_a_block_of_experts_trains():
    """Routing, both experts' products, the activation function between them and the weighted sum, forward and backward, against 64 bits."""
    g = torch.Generator(device="cuda").manual_seed(3)
    E, h, f, T = 6, 64, 96, 150
    make = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x, scores, w1, w2, b1, dy = make(T, h).to(B), make(T, E), (make(E, f, h) / 8).to(B), (make(E, h, f) / 10).to(B), (make(E, f) / 10).to(B), make(T, h)
    leaves = [t.requires_grad_() for t in (x, w1, w2, b1, scores)]
    out = _block(x, scores, w1, w2, b1)
    grads = torch.autograd.grad(out, leaves, dy)
    d = [t.detach().double().requires_grad_() for t in leaves]
    X, W1, W2, B1, S = d
    p = torch.softmax(S, 1)
    chosen = torch.softmax(scores.float(), 1).topk(2, 1).indices
    mask = torch.zeros(T, E, dtype=torch.bool, device="cuda").scatter_(1, chosen, True)
    hid = torch.einsum("th,efh->tef", X, W1) + B1
    every = torch.einsum("tef,ehf->teh", hid * torch.sigmoid(hid), W2)
    want = (every * (p * mask)[:, :, None]).sum(1)
    exact = torch.autograd.grad(want, d, dy.double())
    # the hidden values, their gradients and the results are rounded to 8 bits (2^-9 each), the kept inputs of the activation function to 4 (2^-4 of its slope's argument)
    for got, ref, tol in ((out, want, 2 ** -6), *zip(grads, exact, (2 ** -4,) * 5)):
        assert (got.double() - ref).norm() <= tol * ref.norm()


@gpu
@pytest.mark.parametrize("tokens", [1, 40])
def test_a_block_of_experts_serves_in_8_bits(tokens):
    g = torch.Generator(device="cuda").manual_seed(4)
    E, h, f = 8, 256, 192
    make = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x, scores, w1, w2 = make(tokens, h).to(B), make(tokens, E), make(E, f, h) / 16, make(E, h, f) / 14
    p1, p2 = i8.pack(w1.view(-1, h)), i8.pack(w2.view(-1, f))
    token, ends, weight, order = _route(scores, 2)
    hid = mx.activation(experts.matmul(x[token], p1, ends), "silu")
    out = experts.matmul(hid, p2, ends)
    expert = torch.repeat_interleave(torch.arange(E, device="cuda"), torch.diff(ends, prepend=ends.new_zeros(1)).long())
    v1, v2 = (i8.unpack(p, torch.float32).double() for p in (p1, p2))
    xs = i8.unpack(i8.pack(x[token]), torch.float32).double()
    want = torch.einsum("rh,rfh->rf", xs, v1.view(E, f, h)[expert])
    assert (experts.matmul(x[token], p1, ends).double() - want).norm() <= 2 ** -8 * want.norm()
    hs = i8.unpack(i8.pack(hid), torch.float32).double()
    want = torch.einsum("rf,rhf->rh", hs, v2.view(E, h, f)[expert])
    assert (out.double() - want).norm() <= 2 ** -8 * want.norm()
