"""Matrices in 8-bit integers and their products.

The references are written from the format and the formulas in 64 bits with numpy: codes and scales are compared bit by bit (a quotient of two 24-bit numbers that
is no half lies further from one than 64 bits round).  A product's sum is a whole number: what is off are its rounding to 32 bits, the scales' product,
their product and the result's own type, half a step each.
"""
import numpy as np
import pytest
import torch

from paper_2504_03662_b200 import binding as gb
from paper_2504_03662_b200 import experts, i8, mx

from .test_mx import DT, HALF, close, f64, numbers, step

gpu = pytest.mark.gpu


def ref_pack(x):
    """(codes, scales) of a float64 matrix of 32-bit numbers."""
    bad = ~np.isfinite(x).all(1)
    x = np.where(bad[:, None], 0.0, x)
    scale = (np.maximum(np.abs(x).max(1), 2.0 ** -100) / 127).astype(np.float32)
    codes = np.rint(x / scale.astype(np.float64)[:, None]).astype(np.int8)
    return codes, np.where(bad, np.float32("nan"), scale)


def lay(codes):
    out = np.zeros((codes.shape[0], i8.pitch(codes.shape[1])), np.int8)
    out[:, :codes.shape[1]] = codes
    return out


def held(codes, scales, device="cuda"):
    return i8.Packed(torch.from_numpy(lay(codes)).to(device), torch.from_numpy(np.asarray(scales, np.float32)).to(device), *codes.shape)


def check_pack(x):
    codes, scales = ref_pack(f64(x))
    p = i8.pack(x)
    assert np.array_equal(p.scales.cpu().numpy(), scales, equal_nan=True)
    assert (p.codes.cpu().numpy() == lay(codes)).all(), np.argwhere(p.codes.cpu().numpy() != lay(codes))[:3]
    return p, codes, scales


# ------------------------------------------------------------------------------------------------- without a GPU

def test_sizes():
    lib = gb.load_library()
    for rows, cols in ((1, 1), (3, 16), (5, 17), (0, 9), (1000, 4097)):
        assert lib.galv_i8_codes_bytes(rows, cols) == rows * i8.pitch(cols)
        assert lib.galv_i8_linear_workspace_bytes(rows, cols) == i8._room(rows, cols) >= rows * (i8.pitch(cols) + 4)
    for rows, cols in ((-1, 5), (5, 0), (2 ** 31, 5), (5, 2 ** 31 - 128)):
        assert lib.galv_i8_codes_bytes(rows, cols) == lib.galv_i8_linear_workspace_bytes(rows, cols) == 0
    assert lib.galv_i8_codes_bytes(2 ** 31 - 129, 2 ** 31 - 129) == (2 ** 31 - 129) * (2 ** 31 - 128)


def test_calls_without_a_context_are_refused():
    lib = gb.load_library()
    assert lib.galv_i8_pack(None, 1, 1, None, 1, 0, None, None, None) == gb.ERR_INVALID_ARG
    assert lib.galv_i8_unpack(None, 1, 1, None, None, None, 1, 0, None) == gb.ERR_INVALID_ARG
    assert lib.galv_i8_matmul(None, 1, 1, 1, 1, *[None] * 7, 1, 0, None) == gb.ERR_INVALID_ARG
    assert lib.galv_i8_linear(None, 1, 1, 1, 1, None, None, 1, None, None, None, None, 1, 0, None, 0, None) == gb.ERR_INVALID_ARG


def _fake(rows=4, cols=64):
    return i8.Packed(torch.zeros(rows, i8.pitch(cols), dtype=torch.int8), torch.zeros(rows), rows, cols)


@pytest.mark.parametrize("call", [
    lambda: i8.pack(torch.zeros(4, 64)),                                           # not on a GPU
    lambda: i8.pack(torch.zeros(4, 64, dtype=torch.float64)),
    lambda: i8.pack(torch.zeros(64)),
    lambda: i8.unpack(_fake()),
    lambda: i8.unpack(_fake(), torch.int32),
    lambda: i8.Packed(torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4), 4, 64),
    lambda: i8.Packed(torch.zeros(4, 63, dtype=torch.int8), torch.zeros(4), 4, 63),      # rows of 64 bytes
    lambda: i8.Packed(torch.zeros(4, 64, dtype=torch.int8), torch.zeros(3), 4, 64),
    lambda: i8.Packed(torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4, dtype=torch.float64), 4, 64),
    lambda: i8.Packed(torch.zeros(4, 128, dtype=torch.int8)[:, ::2], torch.zeros(4), 4, 64),
    lambda: i8.Packed(torch.zeros(400, dtype=torch.int8)[1:], torch.zeros(4), 4, 64),    # off 16 bytes
    lambda: i8.Packed(torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4), 4, 0),
    lambda: i8.matmul(_fake(), _fake()),                                           # not on a GPU
    lambda: i8.matmul(_fake(), _fake(4, 65)),
    lambda: i8.matmul(_fake(), _fake(0, 64)),
    lambda: i8.matmul(_fake(), _fake(), torch.int8),
    lambda: i8.matmul(_fake(), _fake(), bias=torch.zeros(4)),
    lambda: i8.matmul(_fake(1, 131072), _fake(1, 131072)),                         # sums could leave 32 bits
    lambda: i8.linear(torch.zeros(4, 63), _fake()),
    lambda: i8.linear(torch.zeros(4, 64, dtype=torch.int8), _fake()),
    lambda: i8.linear(torch.zeros(4, 64), _fake(), torch.zeros(5)),
    lambda: mx.linear(torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(8, 64, dtype=torch.bfloat16), four=True, eight=True),
    lambda: mx.linear(torch.zeros(1, 131072, dtype=torch.bfloat16), torch.zeros(1, 131072, dtype=torch.bfloat16), eight=True),
    lambda: mx.linear(torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(8, 64, dtype=torch.bfloat16), torch.zeros((), dtype=torch.bfloat16), eight=True),
])
def test_refusals(call):
    with pytest.raises(ValueError):
        call()


# ------------------------------------------------------------------------------------------------- packing

@gpu
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 16), (1, 8192), (3, 17), (9, 2048), (7, 2049), (300, 1000), (2, 16384), (3, 16385), (400, 9000), (310, 20000), (2, 32769), (2, 40011), (1000, 7), (2500, 33)])
def test_pack_and_unpack(rows, cols, dtype):
    for pad in (0, 8, 5):
        x = numbers(rows * 7 + cols + pad, rows, cols, DT[dtype], pad)
        wide = x.as_strided((rows, cols + pad), (cols + pad, 1)).cuda()
        p, codes, scales = check_pack(wide[:, :cols])
        want = codes * scales.astype(np.float64)[:, None]
        for out in DT:
            close(i8.unpack(p, DT[out]), want, HALF * np.abs(want) + step(DT[out], want), out)


@gpu
def test_quotients_next_to_a_half():
    """Ties, and the numbers next to them on both sides, under scales that are powers of two and under others."""
    rows = []
    for top in (127.0, 127 * 2.0 ** -9, 1.0, 3.3, 100.1, 9.7e-12, 2.0 ** -99, 1.17e30):
        top = np.float32(top)
        s = np.float32(top / np.float32(127))
        half = ((np.arange(-127, 127) + 0.5) * float(s)).astype(np.float32)
        for x in (half, np.nextafter(half, np.float32(np.inf)), np.nextafter(half, np.float32(-np.inf)), half * np.float32(1 + 2.0 ** -22), half * np.float32(1 - 2.0 ** -22)):
            rows.append(np.concatenate([[top], x, [-top]]))
    check_pack(torch.from_numpy(np.stack(rows).astype(np.float32)).cuda())
    g = np.random.default_rng(3)
    s = (np.abs(g.standard_normal((4000, 1))) + 0.01).astype(np.float32)
    half = ((g.integers(-127, 127, (4000, 200)) + 0.5) * s.astype(np.float64)).astype(np.float32)
    check_pack(torch.from_numpy(np.concatenate([half, 127 * s], 1).astype(np.float32)).cuda())


@gpu
def test_pack_the_ends_of_the_range():
    big, inf, nan = torch.finfo(torch.float32).max, float("inf"), float("nan")
    x = torch.zeros(9, 3000)
    for i, v in enumerate([[big, -big, 1.0], [2.0 ** -149, 0.0, -2.0 ** -140], [0.0, -0.0, 0.0], [2.0 ** -100, 2.0 ** -101, 2.0 ** -108], [inf, 1.0, 2.0], [1.0, nan, 2.0], [-inf, inf, nan],
                           [1e-30, 2e-30, -3e-30], [65504.0, -1.0, 300.0]]):
        x[i, [0, 2047, 2999]] = torch.tensor(v)
    p, codes, scales = check_pack(x.cuda())
    assert torch.isnan(p.scales[4:7]).all() and not p.codes[4:7].any()
    got = i8.unpack(p, torch.float32)
    assert torch.isnan(got[4:7]).all() and torch.isfinite(got[[0, 1, 2, 3, 7, 8]]).all()
    assert not torch.isinf(i8.unpack(p, torch.float16)).any()


# ------------------------------------------------------------------------------------------------- products

def _held_numbers(seed, rows, cols):
    g = np.random.default_rng(seed)
    codes = g.integers(-127, 128, (rows, cols)).astype(np.int8)
    scales = np.exp2(g.uniform(-12, 3, rows)).astype(np.float32)
    return held(codes, scales), codes, scales


def _want(a, sa, b, sb, bias):
    sums = a.astype(np.float64) @ b.astype(np.float64).T                            # exact: below 2^53
    want = sums * sa.astype(np.float64)[:, None] * sb.astype(np.float64)
    return (want if bias is None else want + f64(bias)), np.abs(want)


def in_range(want, dtype):
    """What to-nearest rounding makes of numbers past a type's range: fp16's infinity from 65520 on."""
    return np.where(np.abs(want) >= 65520, np.copysign(np.inf, want), want) if dtype == torch.float16 else want


SHAPES = [(1, 1, 1), (1, 16, 8192), (2, 1000, 96), (5, 33, 100), (16, 256, 4096), (33, 1000, 5003), (64, 2300, 512), (65, 130, 129), (255, 257, 127), (300, 513, 1000), (700, 300, 2048), (1500, 1030, 260)]


@gpu
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_products(m, n, k, dtype):
    (a, av, sa), (b, bv, sb) = _held_numbers(m + k, m, k), _held_numbers(n + k + 1, n, k)
    for with_bias in (False, True):
        bias = numbers(3, 1, n, DT[dtype])[0].cuda() if with_bias else None
        want, size = _want(av, sa, bv, sb, bias)
        got = i8.matmul(a, b, DT[dtype], bias)
        with np.errstate(invalid="ignore"):                                         # infinity less infinity, which are equal
            close(got, in_range(want, DT[dtype]), 3 * HALF * size + 2 * HALF * np.abs(want) + step(DT[dtype], want))
        assert torch.equal(got, i8.matmul(a, b, DT[dtype], bias))


@gpu
def test_sums_are_exact():
    """Of scales one in fp32: as whole numbers below 2^24, and at the largest sums there are (rounded to 24 bits)."""
    g = np.random.default_rng(1)
    a, b = g.integers(-10, 11, (70, 3000)).astype(np.int8), g.integers(-10, 11, (300, 3000)).astype(np.int8)
    got = i8.matmul(held(a, np.ones(70)), held(b, np.ones(300)), torch.float32)
    assert (f64(got) == a.astype(np.float64) @ b.astype(np.float64).T).all()
    k = gb.I8_MOST
    a, b = np.full((3, k), -128, np.int8), np.full((2, k), -128, np.int8)
    b[1] = 127
    got = f64(i8.matmul(held(a, np.ones(3)), held(b, np.ones(2)), torch.float32))
    assert (got == np.float32([k * 16384.0, -128.0 * 127 * k])).all()


@gpu
def test_what_lies_behind_a_rows_end_is_not_read():
    for m in (5, 100):                                                              # both kernels
        (a, av, sa), (b, bv, sb) = _held_numbers(1, m, 300), _held_numbers(2, 290, 300)
        clean = i8.matmul(a, b, torch.float32)
        a.codes[:, 300:], b.codes[:, 300:] = 77, -5
        assert torch.equal(i8.matmul(a, b, torch.float32), clean)


@gpu
def test_rows_that_are_no_numbers():
    """A row with a NaN for its scale gives NaN in its own results alone."""
    (a, av, sa), (b, bv, sb) = _held_numbers(1, 40, 300), _held_numbers(2, 290, 300)
    clean = i8.matmul(a, b, torch.float32)
    a.scales[7], b.scales[280] = float("nan"), float("nan")
    got = i8.matmul(a, b, torch.float32)
    assert torch.isnan(got[7]).all() and torch.isnan(got[:, 280]).all()
    keep = torch.ones_like(got, dtype=torch.bool)
    keep[7], keep[:, 280] = False, False
    assert torch.equal(got[keep], clean[keep])


@gpu
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("shape,n", [((2048,), 500), ((1, 100), 33), ((3, 5, 777), 256), ((0, 64), 8), ((300, 5001), 70)])
def test_linear_is_pack_and_product(shape, n, dtype):
    x = numbers(5, int(np.prod(shape[:-1])), shape[-1], DT[dtype]).reshape(shape).cuda()
    w = i8.pack(numbers(6, n, shape[-1], torch.float32).cuda())
    bias = numbers(7, 1, n, DT[dtype])[0].cuda()
    got = i8.linear(x, w, bias)
    assert got.shape == (*shape[:-1], n)
    flat = x.reshape(-1, shape[-1])
    if flat.shape[0]:
        assert torch.equal(got.reshape(-1, n), i8.matmul(i8.pack(flat), w, DT[dtype], bias))
    wide = torch.full((flat.shape[0], shape[-1] + 3), float("nan"), dtype=DT[dtype], device="cuda")
    wide[:, :shape[-1]] = flat
    assert torch.equal(i8.linear(wide[:, :shape[-1]], w, bias), got.reshape(-1, n))
    assert torch.equal(i8.linear(flat.t().contiguous().t(), w, bias), got.reshape(-1, n))


@gpu
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("m,n,k", [(1, 8192, 8192), (2, 130, 16384), (16, 1000, 8192), (17, 300, 4100), (33, 129, 2050), (48, 2000, 2048), (64, 130, 4096), (64, 5000, 777), (7, 40, 131071), (64, 9000, 8192)])
def test_few_rows(m, n, k, dtype):
    """Up to 64 rows, in clusters of one to eight CTAs: packed in the call as by themselves, a row that is no number among them."""
    x = numbers(m + n, m, k + 1, DT[dtype])
    x[:, 1 + (7919 * m) % k] *= 40
    x[m // 2, k // 3:] = 0
    x[m - 1, k] = float("nan") if m > 1 else 3
    x = x.cuda()
    w = held(*_held_numbers(n, n, k)[1:])
    for rows in (x[:, 1:], x[:, 1:].contiguous()):
        got = i8.linear(rows, w)
        want = i8.matmul(i8.pack(rows), w, DT[dtype])
        assert torch.equal(got.nan_to_num(7.0, 8.0, 9.0), want.nan_to_num(7.0, 8.0, 9.0))
        assert torch.isnan(got[m - 1]).all() == (m > 1) and not torch.isnan(got[:m - 1]).any()
    ends = torch.tensor([0, m // 3, m // 3, m - m // 4], dtype=torch.int32, device="cuda")
    if n % 4 == 0:                                                                  # the same weights as four experts', rows behind the last end
        assert torch.equal(experts.matmul(rows, w, ends).nan_to_num(7.0, 8.0, 9.0), experts.matmul(i8.pack(rows), w, ends, dtype=DT[dtype]).nan_to_num(7.0, 8.0, 9.0))


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_differentiable_linear(dtype):
    x, w, b = (numbers(s, r, c, DT[dtype]).cuda().requires_grad_() for s, r, c in ((1, 200, 300), (2, 130, 300), (3, 1, 130)))
    dy = numbers(4, 200, 130, DT[dtype]).cuda()
    bias = b[0]
    y = mx.linear(x, w, bias, eight=True)
    assert torch.equal(y, i8.matmul(i8.pack(x.detach()), i8.pack(w.detach()), DT[dtype], bias.detach()))
    grads = torch.autograd.grad(y, (x, w, b), dy)
    plain = torch.autograd.grad(mx.linear(x, w, b[0]), (x, w, b), dy)              # straight through the rounding
    assert all(torch.equal(g, p) for g, p in zip(grads, plain))
    with torch.autocast("cuda", dtype=torch.float16):
        assert torch.equal(mx.linear(x, w, bias, eight=True), y)


@gpu
def test_captured_with_other_inputs_and_on_another_stream():
    w = i8.pack(numbers(1, 700, 1000, torch.float32).cuda())
    xs = [numbers(s, 37, 1000, torch.bfloat16).cuda() for s in (2, 3)]
    want = [i8.linear(x, w) for x in xs]
    static = xs[0].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        assert torch.equal(i8.linear(static, w), want[0])
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = i8.linear(static, w)
    for k in (1, 0, 1):
        static.copy_(xs[k])
        graph.replay()
        assert torch.equal(got, want[k])
    mx.check(0)
