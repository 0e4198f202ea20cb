"""Microscaled operators: packing, restoring, the gradients that read what was kept in 8 bits, products in 4 bits.

The references here are written from the format and the formulas in 64 bits with numpy and share nothing with the kernels.  Codes and
scale bytes are compared bit by bit.  Tolerances count roundings: half a step of the output's type, `finfo.eps / 2` of the value, and for the
32-bit arithmetic inside 2^-24 a rounding (2^-23 an addition of a tensor core, which may cut instead of round) times the sum of the
magnitudes that are added.
"""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2504_03662_b200 import binding as gb
from paper_2504_03662_b200 import mx

gpu = pytest.mark.gpu
HALF = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
GRID = {8: np.array([m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8) if (e, m) != (15, 7)]),
        4: np.array([0, .5, 1, 1.5, 2, 3, 4, 6])}


def ref_pack(x, fmt):
    """(codes [rows, nb*32], scale bytes [rows, nb], values [rows, cols]) of a float64 matrix, by search among the format's elements."""
    rows, cols = x.shape
    nb = -(-cols // 32)
    p = np.zeros((rows, nb * 32))
    p[:, :cols] = x
    p = p.reshape(rows, nb, 32)
    bad = ~np.isfinite(p).all(2)
    p = np.where(bad[:, :, None], 0.0, p)
    grid = GRID[fmt]
    amax = np.abs(p).max(2)
    k = np.full(amax.shape, -127)
    for e in range(-127, 128):                              # smallest exponent that takes the block
        k = np.where(amax > grid[-1] * 2.0 ** float(e), e + 1, k)
    v = np.abs(p) / 2.0 ** k[:, :, None].astype(np.float64)
    at = np.clip(np.searchsorted(grid, v), 1, len(grid) - 1)
    lo, hi = grid[at - 1], grid[at]
    up = (v - lo > hi - v) | ((v - lo == hi - v) & (at % 2 == 0))      # ties to the even element: its index is its code
    code = np.where(up, at, at - 1)
    values = grid[code] * 2.0 ** k[:, :, None].astype(np.float64) * np.where(np.signbit(p), -1, 1)
    code = code | (np.signbit(p).astype(int) << (fmt - 1))
    code = np.where(bad[:, :, None], 0, code)
    values = np.where(bad[:, :, None], np.nan, values)
    byte = np.where(bad, 255, k + 127)
    return code.reshape(rows, -1), byte, values.reshape(rows, -1)[:, :cols]


def lay(code, byte, fmt):
    rows, nb = byte.shape
    if fmt == 8:
        out = np.zeros((rows, -(-nb // 16) * 16), np.uint8)
        out[:, :nb] = byte
        return code.astype(np.uint8).reshape(-1), out.reshape(-1)
    out = np.zeros(-(-rows // 128) * -(-nb // 4) * 512, np.uint8)
    r, b = np.meshgrid(np.arange(rows), np.arange(nb), indexing="ij")
    out[(r // 128 * -(-nb // 4) + b // 4) * 512 + r % 32 * 16 + r // 32 % 4 * 4 + b % 4] = byte
    return (code[:, 0::2] | code[:, 1::2] << 4).astype(np.uint8).reshape(-1), out


def numbers(seed, rows, cols, dtype, pad=0, spread=3):
    """Numbers of many sizes, halves of steps among them, as a view of a wider matrix where pad > 0."""
    g = np.random.default_rng(seed)
    x = g.standard_normal((rows, cols)) * 2.0 ** g.integers(-spread, spread + 1, (rows, 1))
    x = np.where(g.random((rows, cols)) < 0.2, np.round(x * 8) / 8, x)
    x[g.random((rows, cols)) < 0.02] = 0
    wide = torch.full((rows, cols + pad), 7.0, dtype=dtype)
    wide[:, :cols] = torch.from_numpy(x).to(dtype)
    return wide[:, :cols]


def f64(t):
    return t.detach().cpu().double().numpy()


def packed(x, fmt, device="cuda"):
    """(Packed on the device from the reference's bytes, its values)."""
    code, byte, values = ref_pack(f64(x), fmt)
    c, s = lay(code, byte, fmt)
    return mx.Packed(torch.from_numpy(c.copy()).to(device), torch.from_numpy(s.copy()).to(device), *x.shape, fmt), values


def close(got, want, tol, what=""):
    got = f64(got)
    bad = ~((np.abs(got - want) <= tol) | (np.isnan(got) & np.isnan(want)) | (got == want))
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: {got[tuple(np.argwhere(bad)[0])]} for {want[tuple(np.argwhere(bad)[0])]}"


def step(dtype, want):
    """Half a step of a type at a value, of its smallest step where it is below the normal numbers."""
    f = torch.finfo(dtype)
    return np.maximum(np.abs(want) * f.eps / 2, f.smallest_normal * f.eps / 2)


# ------------------------------------------------------------------------------------------------- without a GPU

def test_sizes_of_codes_and_scales():
    lib = gb.load_library()
    for rows, cols in ((1, 1), (1, 32), (3, 33), (128, 128), (129, 129), (1000, 4097), (0, 5)):
        nb = -(-cols // 32)
        for fmt in (8, 4):
            code, byte, _ = ref_pack(np.ones((rows, cols)), fmt) if rows else (np.zeros((0, nb * 32), int), np.zeros((0, nb), int), None)
            c, s = lay(code, byte, fmt)
            assert lib.galv_mx_codes_bytes(rows, cols, fmt) == mx.codes_bytes(rows, cols, fmt) == c.size
            assert lib.galv_mx_scales_bytes(rows, cols, fmt) == mx.scales_bytes(rows, cols, fmt) == s.size
    for rows, cols, fmt in ((-1, 5, 8), (5, 0, 8), (5, 5, 6), (2 ** 31, 5, 8), (5, 2 ** 31 - 128, 4)):
        assert lib.galv_mx_codes_bytes(rows, cols, fmt) == 0 and lib.galv_mx_scales_bytes(rows, cols, fmt) == 0
    assert lib.galv_mx_codes_bytes(2 ** 31 - 129, 2 ** 31 - 129, 8) == (2 ** 31 - 129) * (2 ** 31 - 128)      # 64-bit sizes


def test_calls_without_a_context_are_refused():
    lib = gb.load_library()
    z = [None] * 20
    assert lib.galv_mx_pack(None, 1, 1, None, 1, 0, 8, None, None, None) == gb.ERR_INVALID_ARG
    assert lib.galv_mx_unpack(None, 1, 1, 8, None, None, None, 1, 0, None) == gb.ERR_INVALID_ARG
    assert lib.galv_mx_act_backward(None, 1, 1, 0, None, None, None, 1, None, 1, 0, None) == gb.ERR_INVALID_ARG
    assert lib.galv_mx_norm_backward(None, 1, 1, 0, 0.0, None, None, None, 1, None, None, 1, 0, None, None, None, 0, None) == gb.ERR_INVALID_ARG
    assert lib.galv_mx_weight_grad(None, 1, 1, 1, None, 1, 1, *z[:4], 1, None, 0, None) == gb.ERR_INVALID_ARG
    assert lib.galv_mx_matmul(None, 1, 1, 1, *z[:6], 1, 0, None, 0, None) == gb.ERR_INVALID_ARG
    assert lib.galv_mx_norm_workspace_bytes(None, 1, 1) == lib.galv_mx_matmul_workspace_bytes(None, 1, 1, 1) == 0
    assert lib.galv_mx_weight_grad_workspace_bytes(None, 1, 1, 1, None, 1) == 0


def test_the_reference_finds_the_elements():
    x = np.array([[448.0, 464.0, -1.0, 0.0, 2.0 ** -9, 1.5 * 2.0 ** -9] + [0.0] * 26 + [np.inf] + [1.0] * 31 + [6.0, 2.5, -3.5, 5.0, .25, .75] + [0.0] * 26])
    code, byte, v = ref_pack(x[:, :32], 8)
    assert byte.tolist() == [[128]] and v[0, :2].tolist() == [448.0, 448.0] and v[0, 2] == -1.0       # 464 is past 448: one exponent more, a tie at 464/2
    code, byte, v = ref_pack(x[:, 32:64], 8)
    assert byte.tolist() == [[255]] and np.isnan(v).all() and not code.any()
    code, byte, v = ref_pack(x[:, 64:], 4)
    assert byte.tolist() == [[127]] and v[0, :6].tolist() == [6.0, 2.0, -4.0, 4.0, 0.0, 1.0]         # ties to the even code


def _fake(rows=4, cols=64, fmt=8):
    return mx.Packed(torch.zeros(mx.codes_bytes(rows, cols, fmt), dtype=torch.uint8), torch.zeros(mx.scales_bytes(rows, cols, fmt), dtype=torch.uint8), rows, cols, fmt)


@pytest.mark.parametrize("call", [
    lambda: mx.pack(torch.zeros(4, 64)),                                           # not on a GPU
    lambda: mx.pack(torch.zeros(4, 64), 6),                                        # no such format
    lambda: mx.pack(torch.zeros(4, 64, dtype=torch.float64)),                      # no such type
    lambda: mx.pack(torch.zeros(64)),                                              # not a matrix
    lambda: mx.unpack(_fake()),
    lambda: mx.Packed(torch.zeros(4, dtype=torch.uint8), torch.zeros(64, dtype=torch.uint8), 4, 64),
    lambda: mx.Packed(torch.zeros(256, dtype=torch.int8), torch.zeros(64, dtype=torch.uint8), 4, 64),
    lambda: mx.act_backward(torch.zeros(4, 64), _fake(), "relu"),
    lambda: mx.act_backward(torch.zeros(4, 63), _fake()),
    lambda: mx.act_backward(torch.zeros(4, 64), _fake(fmt=4)),
    lambda: mx.norm_backward(torch.zeros(4, 64), _fake(), kind="batch"),
    lambda: mx.norm_backward(torch.zeros(4, 64), _fake(), torch.ones(63)),
    lambda: mx.norm_backward(torch.zeros(4, 64), _fake(), torch.ones(64, dtype=torch.float16)),
    lambda: mx.weight_grad(torch.zeros(4, 8), _fake()),                            # 32-bit gradients
    lambda: mx.weight_grad(torch.zeros(5, 8, dtype=torch.bfloat16), _fake()),
    lambda: mx.weight_grad(torch.zeros(4, 8, dtype=torch.bfloat16), _fake(), torch.float16),
    lambda: mx.weight_grad(torch.zeros(4, 8, dtype=torch.bfloat16), _fake(), base=torch.zeros(8, 63, dtype=torch.bfloat16)),
    lambda: mx.matmul(_fake(), _fake()),                                           # 8 bits
    lambda: mx.matmul(_fake(fmt=4), _fake(4, 96, 4)),
    lambda: mx.matmul(_fake(fmt=4), _fake(fmt=4), bias=torch.zeros(4)),
    lambda: mx.linear(torch.zeros(4, 64), torch.zeros(8, 64)),
    lambda: mx.linear(torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(8, 63, dtype=torch.bfloat16)),
    lambda: mx.linear(torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(0, 64, dtype=torch.bfloat16)),      # no such weight gradient
    lambda: mx.norm(torch.zeros(4, 64), bias=torch.zeros(64), kind="rms"),
    lambda: mx.norm(torch.zeros(4, 64), torch.ones(64, dtype=torch.bfloat16)),      # would only show in the backward pass
    lambda: mx.activation(torch.zeros(4, 64), "relu"),
])
def test_refusals(call):
    with pytest.raises(ValueError):
        call()


# ------------------------------------------------------------------------------------------------- packing

SIZES = [(1, 1), (1, 32), (1, 2048), (2, 31), (3, 33), (5, 100), (127, 96), (128, 128), (129, 160), (300, 513), (64, 1000), (1000, 7)]


@gpu
@pytest.mark.parametrize("fmt", [8, 4])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows,cols", SIZES)
def test_pack_and_unpack(rows, cols, dtype, fmt):
    for pad in (0, 8, 5):
        x = numbers(rows * 7 + cols + pad, rows, cols, DT[dtype], pad)
        code, byte, values = ref_pack(f64(x), fmt)
        c, s = lay(code, byte, fmt)
        wide = x.as_strided((rows, cols + pad), (cols + pad, 1)).cuda()
        p = mx.pack(wide[:, :cols], fmt)
        assert (p.scales.cpu().numpy() == s).all() and (p.codes.cpu().numpy() == c).all()
        for out, to in DT.items():
            got = mx.unpack(p, to)
            want = torch.from_numpy(values).to(to)                 # 8 bits hold the elements exactly; fp16 may have to round small ones
            if to == torch.float16:
                want = torch.from_numpy(np.clip(values, -65504, 65504)).to(to)
            assert torch.equal(got.cpu(), want), out


@gpu
@pytest.mark.parametrize("fmt", [8, 4])
def test_pack_the_ends_of_the_range(fmt):
    big = torch.finfo(torch.float32).max
    tiny = 2.0 ** -149
    rows = [[big, -big, 1.0], [tiny, -tiny, 0.0], [0.0, -0.0, 0.0], [2.0 ** -126, 2.0 ** -130, -2.0 ** -127], [1e-38, 3e-39, -5e-40],
            [448.0, 449.0, 464.0], [6.0, 6.0000005, -6.0], [float("inf"), 1.0, 2.0], [1.0, float("nan"), -float("inf")], [65504.0, 1.0, -65504.0]]
    x = torch.zeros(len(rows), 70)
    x[:, 30:33] = torch.tensor(rows)                               # across two blocks; the third stays zero
    code, byte, values = ref_pack(f64(x), fmt)
    c, s = lay(code, byte, fmt)
    p = mx.pack(x.cuda(), fmt)
    assert (p.scales.cpu().numpy() == s).all() and (p.codes.cpu().numpy() == c).all()
    got = mx.unpack(p, torch.float32).cpu()
    want = torch.from_numpy(values).float()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(0), want.nan_to_num(0))
    assert torch.isnan(got[7, :32]).all() and not torch.isnan(got[7, 32:]).any()
    half = mx.unpack(p, torch.float16).cpu()
    assert not torch.isinf(half).any()                             # what was held as a number stays one


@gpu
def test_every_element_survives():
    """Each code under each scale that holds it comes back as itself."""
    for fmt in (8, 4):
        g = GRID[fmt]
        x = torch.tensor(np.concatenate([g, -g])).double()
        x = x[:, None].repeat(1, 32)
        x[:, 1] = g[-1]                                            # the block's largest fixes its scale
        for k in (-100, -7, 0, 3, 90):
            v = (x * 2.0 ** k).float().cuda()
            assert torch.equal(mx.unpack(mx.pack(v, fmt), torch.float32), v)


@gpu
def test_bytes_around_the_results_stay():
    rows, cols = 37, 100
    galv = mx.context(torch.device("cuda", 0))
    for fmt in (8, 4):
        x = numbers(3, rows, cols, torch.float32).cuda()
        nc, ns = mx.codes_bytes(rows, cols, fmt), mx.scales_bytes(rows, cols, fmt)
        room = torch.full((nc + 512,), 0xA5, dtype=torch.uint8, device="cuda"), torch.full((ns + 512,), 0xA5, dtype=torch.uint8, device="cuda")
        galv.galv_mx_pack(x, fmt, room[0][256:256 + nc], room[1][256:256 + ns])
        for r, n in zip(room, (nc, ns)):
            assert (r[:256] == 0xA5).all() and (r[256 + n:] == 0xA5).all()
        wide = torch.full((rows + 2, cols + 9), 5.0, device="cuda")
        galv.galv_mx_unpack(fmt, room[0][256:256 + nc], room[1][256:256 + ns], wide[1:-1, :cols])
        assert (wide[0] == 5).all() and (wide[-1] == 5).all() and (wide[:, cols:] == 5).all()


# ------------------------------------------------------------------------------------------------- activation functions

def slope(x, act):
    from scipy.special import erf
    if act == "gelu":
        return 0.5 * (1 + erf(x / np.sqrt(2))) + x * np.exp(-x * x / 2) / np.sqrt(2 * np.pi)
    if act == "gelu_tanh":
        k = np.sqrt(2 / np.pi)
        t = np.tanh(k * (x + 0.044715 * x ** 3))
        return 0.5 * (1 + t) + 0.5 * x * (1 - t * t) * k * (1 + 3 * 0.044715 * x * x)
    s = 1 / (1 + np.exp(-np.clip(x, -700, 700)))
    return s * (1 + x * (1 - s))


@gpu
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 2048, 0), (3, 33, 0), (17, 100, 4), (64, 513, 7), (200, 256, 8)])
def test_act_backward(rows, cols, pad, dtype, act):
    kept, x = packed(numbers(1, rows, cols, torch.float32), 8)
    dy = numbers(2, rows, cols, DT[dtype], pad)
    want = f64(dy) * slope(x, act)
    # the slope is a sum of at most two terms up to 1.3 in magnitude, each of functions good to a few 32-bit steps: 16 half steps of 1.3 in all
    tol = np.abs(f64(dy)) * 21 * HALF + step(DT[dtype], want)
    wide = dy.as_strided((rows, cols + pad), (cols + pad, 1)).cuda()
    got = mx.act_backward(wide[:, :cols], kept, act)
    close(got, want, tol, act)
    galv = mx.context(torch.device("cuda", 0))                      # in place
    galv.galv_mx_act_backward(mx.ACTS[act], kept.codes, kept.scales, wide[:, :cols], wide[:, :cols])
    assert torch.equal(wide[:, :cols], got) and (wide[:, cols:] == 7).all()


@gpu
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("dtype,pad", [("bf16", 0), ("f16", 3)])
def test_act_backward_of_large_matrices(dtype, pad, act):
    """Sizes at which slopes are looked up, powers of two inside and outside the table; the slope in 64 bits by torch on the device."""
    g = torch.Generator(device="cuda").manual_seed(3)
    rows, cols = 4000, 8200
    x = torch.randn(rows, cols, generator=g, device="cuda") * torch.exp2(torch.arange(rows, device="cuda").remainder(61).float() - 40)[:, None]
    kept = mx.pack(x)
    v = mx.unpack(kept, torch.float32).double()
    wide = torch.randn(rows, cols + pad, generator=g, device="cuda").to(DT[dtype])
    dy = wide[:, :cols]
    if act == "silu":
        s = torch.sigmoid(v)
        slope64 = s * (1 + v * (1 - s))
    elif act == "gelu":
        slope64 = torch.special.ndtr(v) + v * torch.exp(-v * v / 2) / np.sqrt(2 * np.pi)
    else:
        k = np.sqrt(2 / np.pi)
        c = v.clamp(-50, 50)
        t = torch.tanh(k * (c + 0.044715 * c ** 3))
        slope64 = 0.5 * (1 + t) + 0.5 * c * (1 - t * t) * k * (1 + 3 * 0.044715 * c * c)
    want = dy.double() * slope64
    f = torch.finfo(DT[dtype])
    tol = dy.double().abs() * 21 * HALF + torch.maximum(want.abs() * f.eps / 2, torch.tensor(f.smallest_normal * f.eps / 2, device="cuda", dtype=torch.float64))
    off = (mx.act_backward(dy, kept, act).double() - want).abs()
    assert (off <= tol).all(), (off - tol).max()


@gpu
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
def test_act_backward_far_out(act):
    x = torch.tensor([[0.0, 1e-30, -1e-30, 5.0, -5.0, 12.0, -12.0, 90.0, -90.0, 1e4, -1e4, 1e18, -1e18, 1e30, -1e30, 3e38, -3e38]]).repeat_interleave(32, 1)
    kept, v = packed(x, 8)
    got = mx.act_backward(torch.ones(1, x.shape[1]).cuda(), kept, act)
    with np.errstate(over="ignore", invalid="ignore", under="ignore"):
        want = np.where(v > 50, 1.0, np.where(v < -50, 0.0, slope(np.clip(v, -50, 50), act)))
    close(got, want, 21 * HALF + step(torch.float32, want), act)
    bad, _ = packed(torch.tensor([[float("nan")] + [1.0] * 40]), 8)
    out = f64(mx.act_backward(torch.ones(1, 41).cuda(), bad, act))
    assert np.isnan(out[0, :32]).all() and np.isfinite(out[0, 32:]).all()


# ------------------------------------------------------------------------------------------------- norms

def norm_ref(x, dy, w, kind, eps):
    mean = x.mean(1, keepdims=True) if kind == "layer" else np.zeros((len(x), 1))
    xc = x - mean
    r = 1 / np.sqrt((xc * xc).mean(1, keepdims=True) + eps)
    xn, g = xc * r, dy * w
    dx = r * (g - (g.mean(1, keepdims=True) if kind == "layer" else 0) - xn * (g * xn).mean(1, keepdims=True))
    return dx, (dy * xn).sum(0), dy.sum(0), xn, g, r, mean


def norm_tolerance(x, dy, xn, g, r, kind, dtype, want):
    """A row's sums go through fewer than 64 additions in a chain (16 columns of a thread, then pairs), the rest through a handful of operations: 96 half
    steps of what each term is made of.  xhat is off by 96 half steps of |xhat| and of the largest |x| / deviation (the subtracted mean)."""
    exn = 96 * HALF * (np.abs(xn) + (np.abs(x).max(1, keepdims=True) * r if kind == "layer" else 0))
    gx = np.abs(g * xn).mean(1, keepdims=True)
    egx = (np.abs(g) * exn).mean(1, keepdims=True) + 96 * HALF * gx
    e = 96 * HALF * (np.abs(g) + np.abs(g).mean(1, keepdims=True)) + exn * gx + np.abs(xn) * egx
    rows = len(x)
    chain = 96 + rows
    return r * e + 96 * HALF * np.abs(want) + step(dtype, want), (np.abs(dy) * exn).sum(0) + chain * HALF * np.abs(dy * xn).sum(0), chain * HALF * np.abs(dy).sum(0)


@gpu
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows,cols,pad,weighted", [(1, 16, 0, True), (1, 2048, 0, False), (3, 33, 0, True), (17, 100, 4, True), (70, 513, 7, True), (200, 256, 8, False),
                                                    (5, 5000, 0, True), (2, 12288, 0, True), (3, 20001, 1, True), (400, 64, 0, True), (1, 70000, 0, True)])
def test_norm_backward(rows, cols, pad, weighted, dtype, kind):
    kept, x = packed(numbers(1, rows, cols, torch.float32, spread=1) + 0.5, 8)
    dy = numbers(2, rows, cols, DT[dtype], pad)
    w = (1 + 0.1 * numbers(3, 1, cols, torch.float32)[0]).to(DT[dtype]) if weighted else None
    wn = f64(w) if weighted else np.ones(cols)
    dx, dw, db, xn, g, r, mean = norm_ref(x, f64(dy), wn, kind, 1e-5)
    tx, tw, tb = norm_tolerance(x, f64(dy), xn, g, r, kind, DT[dtype], dx)
    wide = dy.as_strided((rows, cols + pad), (cols + pad, 1)).cuda()
    wc = None if w is None else w.cuda()
    gx, gw, gbias = mx.norm_backward(wide[:, :cols], kept, wc, kind)
    close(gx, dx, tx, "dx")
    close(gw, dw, tw, "dweight")
    if kind == "layer":
        close(gbias, db, tb, "dbias")
    else:
        assert gbias is None
    # the same bits again, and in place
    galv = mx.context(torch.device("cuda", 0))
    ws = torch.empty(max(256, galv.galv_mx_norm_workspace_bytes(rows, cols)), dtype=torch.uint8, device="cuda")
    gw2 = torch.full((cols,), 9.0, device="cuda")
    galv.galv_mx_norm_backward(mx.NORMS[kind], 1e-5, kept.codes, kept.scales, wide[:, :cols], wc, wide[:, :cols], gw2, None, ws)
    assert torch.equal(wide[:, :cols], gx) and torch.equal(gw2, gw) and (wide[:, cols:] == 7).all()


@gpu
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("dtype,rows,cols,pad", [("f32", 300, 12008, 0), ("f32", 77, 16384, 3), ("f32", 2, 16385, 0), ("bf16", 230, 16390, 1), ("f16", 75, 32768, 0), ("f16", 100, 32769, 7),
                                                 ("bf16", 33, 65536, 0), ("bf16", 2, 65537, 0)])
def test_norm_backward_of_shared_rows(dtype, rows, cols, pad, kind):
    """Rows that two or four CTAs share, several a cluster, and both sides of the widths where the way changes."""
    test_norm_backward(rows, cols, pad, True, dtype, kind)


@gpu
def test_norm_backward_of_odd_rows():
    x = torch.ones(4, 64)
    x[1] = 0
    x[2, 3] = float("nan")
    x[3] = torch.arange(64).float()
    kept, v = packed(x, 8)
    dy = torch.ones(4, 64)
    dy[:, ::2] = 2
    dx, dw, db = mx.norm_backward(dy.cuda(), kept, None, "layer", 1e-5)
    assert torch.isfinite(dx[:2]).all() and torch.isfinite(dx[3]).all() and torch.isnan(dx[2]).all()      # equal rows have 1/sqrt(eps), a NaN its row
    want = norm_ref(v[:1], f64(dy[:1]), np.ones(64), "layer", 1e-5)[0]
    close(dx[:1], want, 96 * HALF * 2 / np.sqrt(1e-5) * np.ones(64))
    assert torch.isnan(dw).all() and torch.isfinite(db).all()
    kept0 = mx.pack(torch.ones(0, 64).cuda())
    dx, dw, db = mx.norm_backward(torch.ones(0, 64).cuda(), kept0)
    assert dx.shape == (0, 64) and (dw == 0).all() and (db == 0).all()


# ------------------------------------------------------------------------------------------------- weight gradients

@gpu
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("tokens,n,k,pad", [(1, 1, 1, 0), (1, 128, 256, 0), (5, 33, 70, 0), (64, 128, 128, 0), (65, 129, 257, 3), (200, 300, 500, 8), (1000, 64, 96, 0),
                                            (63, 520, 40, 0), (300, 1, 300, 1), (300, 300, 1, 0), (700, 256, 512, 0)])
def test_weight_grad(tokens, n, k, pad, dtype, out):
    kept, x = packed(numbers(1, tokens, k, torch.float32), 8)
    dy = numbers(2, tokens, n, DT[dtype], pad)
    xt = f64(torch.from_numpy(np.clip(x, -65504, 65504) if dtype == "f16" else x).to(DT[dtype]))
    want = f64(dy).T @ xt
    tol = (tokens / 16 + 4) * 2 * HALF * (np.abs(f64(dy)).T @ np.abs(xt))
    wide = dy.as_strided((tokens, n + pad), (n + pad, 1)).cuda()
    got = mx.weight_grad(wide[:, :n], kept, DT[out])
    close(got, want, tol + step(DT[out], want))
    assert torch.equal(got, mx.weight_grad(wide[:, :n], kept, DT[out]))                       # the same bits again
    base = numbers(3, n, k, DT[out]).cuda()
    sum_ = f64(base) + want
    res = mx.weight_grad(wide[:, :n], kept, base=base)
    close(res, sum_, tol + HALF * np.abs(sum_) + HALF * np.abs(want) + step(DT[out], sum_))
    keep = base.clone()
    assert mx.weight_grad(wide[:, :n], kept, base=base, out=base) is base and torch.equal(base, res) and not torch.equal(base, keep)
    assert (wide[:, n:] == 7).all()


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_weight_grad_of_nothing_and_of_odd_values(dtype):
    empty = mx.pack(torch.zeros(0, 40, device="cuda"))
    dy = torch.zeros(0, 24, dtype=DT[dtype], device="cuda")
    assert (mx.weight_grad(dy, empty) == 0).all()
    base = numbers(3, 24, 40, torch.float32).cuda()
    assert torch.equal(mx.weight_grad(dy, empty, base=base), base)
    x = torch.ones(3, 100)
    x[1, 40] = float("inf")                                        # its block of 32 stands for NaN
    x[2, 90] = 3e38 if dtype == "bf16" else 1e30
    kept, v = packed(x, 8)
    dy = torch.ones(3, 9, dtype=DT[dtype]).cuda()
    got = f64(mx.weight_grad(dy, kept, torch.float32))
    assert np.isnan(got[:, 32:64]).all() and np.isfinite(got[:, :32]).all() and np.isfinite(got[:, 64:]).all()
    assert np.allclose(got[:, 90], 65506.0 if dtype == "f16" else v[2, 90], rtol=1e-6)
    small = torch.full((2, 32), 2.0 ** -20)                          # below fp16's normal numbers, and held exactly
    kept, v = packed(small, 8)
    dy = torch.ones(2, 3, dtype=DT[dtype]).cuda()
    assert (f64(mx.weight_grad(dy, kept, torch.float32)) == 2.0 ** -19).all()


# ------------------------------------------------------------------------------------------------- products

@gpu
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 256, 512), (3, 33, 70), (7, 1000, 1024), (16, 130, 96), (33, 128, 128), (64, 64, 2048), (128, 128, 256), (129, 257, 300), (200, 513, 160),
                                   (300, 520, 1000), (1, 4096, 4096), (513, 1, 64)])
def test_matmul(m, n, k, dtype):
    (a, av), (b, bv) = packed(numbers(1, m, k, torch.float32), 4), packed(numbers(2, n, k, torch.float32), 4)
    want = av @ bv.T
    tol = (k / 32 + 4) * 2 * HALF * (np.abs(av) @ np.abs(bv).T)
    got = mx.matmul(a, b, DT[dtype])
    close(got, want, tol + step(DT[dtype], want))
    assert torch.equal(got, mx.matmul(a, b, DT[dtype]))
    bias = numbers(3, 1, n, DT[dtype])[0].cuda()
    want = want + f64(bias)
    close(mx.matmul(a, b, DT[dtype], bias), want, tol + HALF * np.abs(want) + step(DT[dtype], want))
    wide = torch.full((m + 2, n + 5), 5.0, dtype=DT[dtype], device="cuda")
    galv = mx.context(torch.device("cuda", 0))
    ws = torch.empty(max(256, galv.galv_mx_matmul_workspace_bytes(m, n, k)), dtype=torch.uint8, device="cuda")
    galv.galv_mx_matmul(k, a.codes, a.scales, b.codes, b.scales, None, wide[1:-1, :n], ws)
    assert torch.equal(wide[1:-1, :n], got) and (wide[0] == 5).all() and (wide[-1] == 5).all() and (wide[:, n:] == 5).all()


@gpu
def test_matmul_of_odd_values():
    x, w = torch.ones(40, 200), torch.ones(70, 200)
    x[3, 100] = float("nan")
    w[5, 7] = float("inf")
    x[7] = 0
    x[8] = 3e38
    w[9] = 1e-38
    (a, av), (b, bv) = packed(x, 4), packed(w, 4)
    got = f64(mx.matmul(a, b, torch.float32))
    nan = np.zeros((40, 70), bool)
    nan[3], nan[:, 5] = True, True
    assert (np.isnan(got) == nan).all()
    with np.errstate(invalid="ignore"):
        want = av @ bv.T
    over = np.abs(want) > 3.4e38
    assert np.isinf(got[over & ~nan]).all()
    fine = ~nan & ~over
    assert np.allclose(got[fine], want[fine], rtol=1e-5, atol=0)
    assert mx.matmul(mx.pack(torch.zeros(0, 64, device="cuda"), 4), mx.pack(torch.ones(3, 64, device="cuda"), 4)).shape == (0, 3)


# ------------------------------------------------------------------------------------------------- refusals of the library, streams, graphs

@gpu
def test_the_library_refuses():
    galv = mx.context(torch.device("cuda", 0))
    lib, h = galv.lib, galv.h
    buf = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    p = buf.data_ptr()
    bad = gb.ERR_INVALID_ARG
    pk = lambda **k: lib.galv_mx_pack(h, k.get("rows", 4), k.get("cols", 64), k.get("x", p), k.get("stride", 64), k.get("dtype", 0), k.get("fmt", 8), k.get("codes", p + 8192),
                                      k.get("scales", p + 16384), None)
    assert pk() == gb.OK and pk(rows=0, x=None) == gb.OK
    for k in (dict(rows=-1), dict(cols=0), dict(stride=63), dict(x=None), dict(x=p + 2), dict(dtype=3), dict(fmt=6), dict(codes=None), dict(codes=p + 8200), dict(scales=p + 16385),
              dict(rows=2 ** 31 - 128)):
        assert pk(**k) == bad, k
        assert b"galv_mx_pack" in lib.galv_last_error(h)
    assert lib.galv_mx_unpack(h, 4, 64, 8, p, p + 8192, p + 16384, 63, 0, None) == bad
    assert lib.galv_mx_act_backward(h, 4, 64, 3, p, p + 8192, p + 16384, 64, p + 32768, 64, 0, None) == bad
    assert lib.galv_mx_act_backward(h, 4, 64, 0, p, p + 8192, p + 16384, 64, p + 16384, 65, 0, None) == bad         # in place with another stride
    nb = lambda kind=0, eps=1e-5, dbias=p + 40960, ws=p + 49152, n=8192: lib.galv_mx_norm_backward(h, 4, 64, kind, eps, p, p + 8192, p + 16384, 64, None, p + 24576, 64, 0, p + 32768, dbias, ws, n, None)
    assert lib.galv_mx_norm_workspace_bytes(h, 4, 64) <= 8192 and nb() == gb.OK
    assert nb(kind=1) == bad and nb(kind=2, dbias=None) == bad and nb(eps=-1.0) == bad and nb(eps=float("nan")) == bad
    many = torch.zeros(4 << 20, dtype=torch.uint8, device="cuda")   # few rows need no workspace, many do
    q = many.data_ptr()
    nm = lambda ws, n: lib.galv_mx_norm_backward(h, 2000, 64, 0, 1e-5, q, q + (1 << 18), q + (1 << 19), 64, None, q + (2 << 20), 64, 0, p, p + 4096, ws, n, None)
    need = lib.galv_mx_norm_workspace_bytes(h, 2000, 64)
    assert 0 < need <= 1 << 20 and nm(q + (3 << 20), need) == gb.OK
    assert nm(None, need) == nm(q + (3 << 20) + 1, need) == nm(q + (3 << 20), need - 1) == gb.ERR_WORKSPACE
    wg = lambda dtype=1, out=1, dy=p, stride=8, ws=p + 49152, n=8192: lib.galv_mx_weight_grad(h, 4, 8, 64, dy, stride, dtype, p + 8192, p + 16384, None, p + 24576, out, ws, n, None)
    assert lib.galv_mx_weight_grad_workspace_bytes(h, 4, 8, 64, p, 8) <= 8192 and wg() == gb.OK
    assert wg(dtype=0, out=0) == bad and wg(dtype=1, out=2) == bad and wg(dy=None) == bad and wg(stride=7) == bad and wg(dy=p + 1) == bad
    mm = lambda m=4, n=8, k=64, y=p + 24576, stride=8, dtype=1: lib.galv_mx_matmul(h, m, n, k, p, p + 8192, p + 16384, p + 20480, None, y, stride, dtype, p + 49152, 8192, None)
    assert lib.galv_mx_matmul_workspace_bytes(h, 4, 8, 64) <= 8192 and mm() == gb.OK and mm(m=0, y=None) == gb.OK
    assert mm(n=0) == mm(k=0) == mm(m=-1) == mm(y=None) == mm(stride=7) == mm(dtype=5) == bad
    torch.cuda.synchronize()
    assert lib.galv_mx_status(None, None) == bad
    galv.galv_mx_status()                                           # no wait has run out


def _everything(x, dy, w4, weight):
    kept = mx.pack(x)
    return [mx.unpack(kept, x.dtype), mx.act_backward(dy, kept), *mx.norm_backward(dy, kept, weight), mx.weight_grad(dy, kept, torch.float32),
            mx.matmul(mx.pack(x, 4), w4, x.dtype)]


def _inputs(seed, rows=96, cols=320):
    x, dy = numbers(seed, rows, cols, torch.bfloat16).cuda(), numbers(seed + 1, rows, cols, torch.bfloat16).cuda()
    return x, dy, mx.pack(numbers(seed + 2, 200, cols, torch.bfloat16).cuda(), 4), numbers(seed + 3, 1, cols, torch.bfloat16)[0].cuda()


@gpu
def test_on_another_stream_and_thread():
    import threading
    args = _inputs(1)
    want = _everything(*args)
    torch.cuda.synchronize()
    got, side = [], torch.cuda.Stream()

    def work():
        with torch.cuda.stream(side):
            torch.cuda._sleep(10_000_000)                          # what runs on the wrong stream would be done before its inputs
            fresh = [args[0].clone(), args[1].clone()]
            got.extend(_everything(*fresh, *args[2:]))
        side.synchronize()

    t = threading.Thread(target=work)
    t.start()
    t.join()
    assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))


@gpu
def test_captured_and_replayed():
    args = _inputs(1)
    other = _inputs(9)
    want = [t.clone() for t in _everything(*args)]
    want2 = [t.clone() for t in _everything(*other)]
    static = [args[0].clone(), args[1].clone(), args[2], args[3].clone()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _everything(*static)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _everything(*static)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    for s, o in ((static[0], other[0]), (static[1], other[1]), (static[2].codes, other[2].codes), (static[2].scales, other[2].scales), (static[3], other[3])):
        s.copy_(o)
    graph.replay()
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(out, want2))


@gpu
def test_offsets_beyond_32_bits():
    """2.15e9 elements: the last rows of everything are what they are on their own."""
    rows, cols, last = 65600, 32800, 80
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(rows, cols, generator=g, device="cuda", dtype=torch.bfloat16)
    tail = x[-last:].clone()
    kept, small = mx.pack(x), mx.pack(tail)
    assert torch.equal(kept.codes[-small.codes.numel():], small.codes) and torch.equal(kept.scales[-small.scales.numel():], small.scales)
    assert torch.equal(mx.unpack(kept)[-last:], mx.unpack(small))
    for act in ("gelu", "silu"):
        got = mx.act_backward(x, kept, act)[-last:].float()
        assert torch.allclose(got, mx.act_backward(tail, small, act).float(), rtol=2 ** -7, atol=1.3e-5)      # looked up or computed: 21 * 2^-24 of |dy| < 5 and half a step each
        del got
    assert torch.equal(mx.norm_backward(x, kept)[0][-last:], mx.norm_backward(tail, small)[0])
    dy = torch.zeros(rows, 16, device="cuda", dtype=torch.bfloat16)
    dy[-last:] = torch.randn(last, 16, generator=g, device="cuda").bfloat16()
    a, b = mx.weight_grad(dy, kept, torch.float32), mx.weight_grad(dy[-last:].contiguous(), small, torch.float32)
    assert torch.allclose(a, b, rtol=1e-5, atol=1e-4)               # tokens in other chunks, other orders: (80 / 16 + 4) * 2^-23 of sums of magnitudes below 90 at most
    four, four_tail = mx.pack(x, 4), mx.pack(tail, 4)
    assert torch.equal(mx.unpack(four)[-last:], mx.unpack(four_tail))
    del x, kept, four
    left, right = mx.pack(torch.randn(rows, 64, generator=g, device="cuda", dtype=torch.bfloat16), 4), mx.pack(torch.randn(cols, 64, generator=g, device="cuda", dtype=torch.bfloat16), 4)
    y = mx.matmul(left, right, torch.float16)
    want = mx.unpack(left, torch.float32)[-last:].double() @ mx.unpack(right, torch.float32).double().t()
    assert ((y[-last:].double() - want).abs() <= want.abs() * 2.0 ** -11 + 1e-6).all()


@gpu
def test_the_widest_weight_gradient():
    """As many columns of dy as the limit allows, off the 16-byte boundary (realigned before the product): one token, so dw is dy times 3, exactly."""
    n = 2 ** 31 - 129
    dy = torch.zeros(n + 1, dtype=torch.bfloat16, device="cuda")[1:].view(1, n)
    dy[:, ::1000003] = 2.0
    dy[:, -300:] = torch.arange(300, device="cuda").to(torch.bfloat16)[None] % 64
    dw = mx.weight_grad(dy, mx.pack(torch.full((1, 1), 3.0, device="cuda")))
    assert dw.shape == (n, 1) and torch.equal(dw.view(1, n), dy.mul_(3))


# ------------------------------------------------------------------------------------------------- a run of them

@gpu
@pytest.mark.parametrize("kind,act,dtype", [("layer", "gelu", "bf16"), ("rms", "silu", "f16"), ("layer", "gelu_tanh", "bf16")])
def test_a_layer_that_keeps_8_bits(kind, act, dtype):
    """norm -> linear -> activation -> linear, forward and backward, against the same chain in 64 bits whose backward reads the held values."""
    d, (rows, h, f) = DT[dtype], (150, 192, 320)
    x = numbers(1, rows, h, d, spread=0).cuda().requires_grad_()
    p = [t.cuda().requires_grad_() for t in ((1 + numbers(2, 1, h, torch.float32)[0] / 10).to(d), (numbers(3, f, h, torch.float32, spread=0) / 14).to(d), (numbers(4, 1, f, torch.float32)[0] / 10).to(d),
                                             (numbers(5, h, f, torch.float32, spread=0) / 18).to(d))]
    nw, w1, b1, w2 = p
    a0 = mx.norm(x.view(3, 50, h), nw, None, kind)
    a1 = mx.linear(a0, w1, b1)
    a2 = mx.activation(a1, act)
    y = mx.linear(a2, w2)
    dy = numbers(6, rows, h, d, spread=0).cuda().view(3, 50, h)
    y.backward(dy)
    X, A0, A1, A2 = (f64(t).reshape(rows, -1) for t in (x, a0, a1, a2))
    hold = lambda t: ref_pack(t, 8)[2]
    g3 = f64(dy).reshape(rows, h)
    # every step takes the rounded result of the one before, so the reference does too: each is off by what its own arithmetic rounds
    r16 = lambda t: f64(torch.from_numpy(t).to(d))
    dw2 = g3.T @ hold(A2)
    g2 = r16(g3 @ f64(w2))
    g1 = r16(g2 * slope(hold(A1), act))
    dw1, db1 = g1.T @ hold(A0), g1.sum(0)
    g0 = r16(g1 @ f64(w1))
    dx, dnw, *_ = norm_ref(hold(X), g0, f64(nw), kind, 1e-5)
    # the references round the chain's gradients once more on their own, which may fall the other way: a whole step of the type each, of the 2-norm
    eps = torch.finfo(d).eps
    for got, want, steps in ((w2.grad, dw2, 1), (w1.grad, dw1, 4), (b1.grad, db1, 4), (nw.grad, dnw, 6), (x.grad, dx, 6)):
        got = f64(got).reshape(want.shape)
        assert np.linalg.norm(got - want) <= steps * eps * np.linalg.norm(want)


@gpu
def test_gradients_against_differences():
    """The gradients are the slopes of the formulas at the held point: inputs that 8 bits hold exactly, central differences in 64 bits."""
    g = np.random.default_rng(5)
    x = torch.from_numpy(g.choice([-2.0, -1.5, -0.75, 0.25, 0.5, 1.0, 1.75, 2.0], (3, 48)))
    x[:, ::32] = 2.0
    kept, v = packed(x, 8)
    assert (v == x.numpy()).all()
    dy, w = g.standard_normal((3, 48)).astype(np.float32).astype(np.float64), 1 + 0.1 * g.standard_normal(48).astype(np.float32).astype(np.float64)

    def value(f, at):
        return (dy * f(at)).sum()

    def f_norm(kind):
        def f(t):
            c = t - t.mean(1, keepdims=True) if kind == "layer" else t
            return c / np.sqrt((c * c).mean(1, keepdims=True) + 1e-5) * w
        return f

    from scipy.special import erf
    f_act = {"gelu": lambda t: t * 0.5 * (1 + erf(t / np.sqrt(2))), "silu": lambda t: t / (1 + np.exp(-t)),
             "gelu_tanh": lambda t: 0.5 * t * (1 + np.tanh(np.sqrt(2 / np.pi) * (t + 0.044715 * t ** 3)))}
    cases = [(f_act[a], mx.act_backward(torch.from_numpy(dy).float().cuda(), kept, a)) for a in f_act]
    cases += [(f_norm(k), mx.norm_backward(torch.from_numpy(dy).float().cuda(), kept, torch.from_numpy(w).float().cuda(), k)[0]) for k in ("layer", "rms")]
    for f, got in cases:
        for r, c in ((0, 0), (0, 17), (1, 31), (2, 32), (2, 47)):
            e = np.zeros_like(v)
            e[r, c] = 1e-5
            want = (value(f, v + e) - value(f, v - e)) / 2e-5
            assert abs(float(got[r, c]) - want) < 1e-4 * max(1, abs(want))


@gpu
def test_linear_in_4_bits():
    x, w, b = (t.cuda() for t in (numbers(1, 60, 96, torch.bfloat16, spread=0), numbers(2, 70, 96, torch.bfloat16, spread=0), numbers(3, 1, 70, torch.bfloat16)[0]))
    w.requires_grad_()
    y = mx.linear(x, w, b, four=True)
    av, bv = ref_pack(f64(x), 4)[2], ref_pack(f64(w), 4)[2]
    want = av @ bv.T + f64(b)
    close(y, want, 7 * 2 * HALF * (np.abs(av) @ np.abs(bv).T + np.abs(f64(b))) + step(torch.bfloat16, want))
    y.backward(torch.ones_like(y))
    want = np.ones((60, 70)).T @ ref_pack(f64(x), 8)[2]
    close(w.grad, want, 8 * 2 * HALF * np.abs(ref_pack(f64(x), 8)[2]).sum(0) + step(torch.bfloat16, want))


@gpu
def test_a_backward_pass_captured():
    x, w = numbers(1, 64, 96, torch.bfloat16).cuda(), numbers(2, 32, 96, torch.bfloat16).cuda().requires_grad_()

    def once():
        return torch.autograd.grad(mx.activation(mx.linear(x, w)).float().sum(), w)[0]

    want = once().clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        once()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = once()
    graph.replay()
    assert torch.equal(got, want)
