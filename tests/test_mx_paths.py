"""Microscaled operators: sizes that take each way through the kernels.

What a way has of its own (clusters, splits, segments, tiles after the first, launches ahead) is reached with numbers everywhere, and results are compared in
full.  Large products are compared with products of the held values in 64 bits on the device (torch), the others with numpy's.  Tolerances as in test_mx.
"""
import numpy as np
import pytest
import torch

from paper_2504_03662_b200 import binding as gb
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


# ------------------------------------------------------------------------------------------------- weight gradients in segments, tiles and splits

def _rows(g, rows, cols, dtype, pad=0):
    """Random numbers, rows of other sizes, as a view of a wider matrix where pad > 0."""
    x = torch.randn(rows, cols + pad, generator=g, device="cuda") * torch.exp2(torch.randint(-2, 3, (rows, 1), generator=g, device="cuda").float())
    return x.to(dtype)[:, :cols]


def _within(got, want, tol, dtype):
    f = torch.finfo(dtype)
    rounding = torch.clamp(want.abs() * (f.eps / 2), min=f.smallest_normal * f.eps / 2)
    off = (got.double() - want).abs()
    assert not torch.isnan(off).any() and (off <= tol + rounding).all(), f"{(off > tol + rounding).sum()} of {off.numel()} off, first at {(off > tol + rounding).nonzero()[0].tolist()}"


@gpu
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f32")])
@pytest.mark.parametrize("tokens,n,k,pad", [(2100, 2400, 2048, 0),      # 80 tiles, not split: 33 chunks in three segments, second tiles of some pairs
                                            (5000, 2050, 2300, 6),      # 81 tiles with ragged ends, five segments, dy on other boundaries
                                            (1025, 2561, 1793, 0),      # 88 tiles, a second segment of one token, odd rows
                                            (3000, 1201, 1275, 3),      # 25 tiles, two splits of two segments each
                                            (9000, 300, 700, 0)])       # 6 tiles, twelve splits of 12 chunks or less
def test_weight_gradients_of_many_tokens(tokens, n, k, pad, dtype, out):
    g = torch.Generator(device="cuda").manual_seed(tokens)
    kept = mx.pack(_rows(g, tokens, k, torch.bfloat16))
    dy = _rows(g, tokens, n, DT[dtype], pad)
    x64, dy64 = mx.unpack(kept, DT[dtype]).double(), dy.double()
    want, magnitude = dy64.t() @ x64, dy64.abs().t() @ x64.abs()
    # a tensor core adds at most 1024 tokens, 16 at a time (a whole step each), registers or splits join them
    tol = (64 + tokens / 1024 + 16) * 2 * HALF * magnitude
    got = mx.weight_grad(dy, kept, DT[out])
    _within(got, want, tol, DT[out])
    assert torch.equal(got, mx.weight_grad(dy, kept, DT[out]))
    base = _rows(g, n, k, DT[out])
    total = base.double() + want
    joined = mx.weight_grad(dy, kept, base=base)
    _within(joined, total, tol + HALF * (total.abs() + want.abs()), DT[out])
    assert mx.weight_grad(dy, kept, base=base, out=base) is base and torch.equal(base, joined)


# ------------------------------------------------------------------------------------------------- products of many tiles, and split ones

@gpu
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("m,n,k", [(2600, 2600, 1100),                  # 121 tiles: pairs take a second one while the first moves out; five chunks fill the ring
                                   (2500, 2305, 4200),                  # 100 tiles of 17 chunks, odd columns
                                   (65, 20000, 700),                    # 79 tiles in one row of them
                                   (200, 2048, 8192),                   # 8 tiles, eight splits
                                   (70, 100, 2048),                     # one tile, two splits
                                   (513, 1001, 3000)])                  # 12 tiles, three splits, odd columns
def test_products_of_many_chunks(m, n, k, dtype):
    g = torch.Generator(device="cuda").manual_seed(m)
    a, b = mx.pack(_rows(g, m, k, torch.bfloat16), 4), mx.pack(_rows(g, n, k, torch.bfloat16), 4)
    a64, b64 = mx.unpack(a, torch.float32).double(), mx.unpack(b, torch.float32).double()
    want, tol = a64 @ b64.t(), (k / 32 + 4) * 2 * HALF * (a64.abs() @ b64.abs().t())
    got = mx.matmul(a, b, DT[dtype])
    _within(got, want, tol, DT[dtype])
    assert torch.equal(got, mx.matmul(a, b, DT[dtype]))
    bias = _rows(g, 1, n, DT[dtype])[0]
    total = want + bias.double()
    _within(mx.matmul(a, b, DT[dtype], bias), total, tol + HALF * total.abs(), DT[dtype])
    galv = mx.context(torch.device("cuda", 0))                          # into rows of a wider matrix, whose rest stays
    wide = torch.full((m + 2, n + 5), 5.0, dtype=DT[dtype], device="cuda")
    ws = torch.full((max(256, galv.galv_mx_matmul_workspace_bytes(m, n, k)),), 0xFF, dtype=torch.uint8, device="cuda")
    galv.galv_mx_matmul(k, a.codes, a.scales, b.codes, b.scales, None, wide[1:-1, :n], ws)
    assert torch.equal(wide[1:-1, :n], got) and (wide[0] == 5).all() and (wide[-1] == 5).all() and (wide[:, n:] == 5).all()


# ------------------------------------------------------------------------------------------------- waits that run out

def _all_look():
    """This thread's context and that of the autograd engine's thread look, whatever they find."""
    x, w = torch.ones(1, 32, device="cuda", dtype=torch.bfloat16), torch.ones(1, 32, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    for call in (lambda: mx.check(0), lambda: mx.linear(x, w).sum().backward()):
        try:
            call()
        except gb.GalvError as e:
            assert e.code == gb.ERR_TIMEOUT


@pytest.fixture
def counted():
    """A function that counts `n` more waits as run out on device 0, as the kernels do; every context has looked before the test and behind it."""
    main = mx.context(torch.device("cuda", 0))

    def more(n):
        main.lib.galv_mx_timeouts(main.h)[0] += n

    _all_look()
    yield more
    _all_look()


def _says_timeout(galv):
    try:
        galv.galv_mx_status()
    except gb.GalvError as e:
        assert e.code == gb.ERR_TIMEOUT and "wait" in str(e)
        return True
    return False


@gpu
def test_each_context_reports_a_wait_that_ran_out_once(counted):
    old = gb.Galv(0)
    before = old.galv_mx_timeouts()
    assert not _says_timeout(old)
    counted(3)
    assert old.galv_mx_timeouts() == before + 3
    fresh = gb.Galv(0)                                              # made behind it: nothing has run out since
    assert not _says_timeout(fresh)
    assert _says_timeout(old) and not _says_timeout(old)
    counted(1)
    assert _says_timeout(fresh) and _says_timeout(old)
    assert not _says_timeout(fresh) and not _says_timeout(old)
    old.close(), fresh.close()


def test_the_count_needs_a_context():
    assert not gb.load_library().galv_mx_timeouts(None)


@gpu
def test_products_raise_behind_a_wait_that_ran_out(counted):
    device = torch.device("cuda", 0)
    x, dy = torch.randn(64, 96, device=device).bfloat16(), torch.randn(64, 32, device=device).bfloat16()
    kept, four = mx.pack(x), mx.pack(x, 4)
    want = mx.weight_grad(dy, kept), mx.matmul(four, four)
    mx.check(device)
    for call in (lambda: mx.weight_grad(dy, kept), lambda: mx.matmul(four, four), lambda: mx.check(device), lambda: mx.check(0)):
        counted(1)
        with pytest.raises(gb.GalvError) as e:
            call()
        assert e.value.code == gb.ERR_TIMEOUT
        call()                                                      # said once
        assert torch.equal(mx.weight_grad(dy, kept), want[0]) and torch.equal(mx.matmul(four, four), want[1])
    # a training step: the backward pass runs in a thread of its own, with a context of its own
    w = torch.randn(32, 96, device=device).bfloat16().requires_grad_()
    _all_look()
    mx.linear(x, w).backward(dy)
    counted(1)
    y = mx.linear(x, w)
    with pytest.raises(gb.GalvError):
        y.backward(dy)
    mx.linear(x, w).backward(dy)


# ------------------------------------------------------------------------------------------------- refusals of the differentiable forms

def _short(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


@pytest.mark.parametrize("call", [
    lambda: mx.linear(_short(4, 64), _short(8, 64), _short(4, 8)),                 # adds up, but has no gradient of this shape
    lambda: mx.linear(_short(4, 64), _short(8, 64), _short(1, 8)),
    lambda: mx.linear(_short(4, 64), _short(8, 64), torch.zeros(8)),
    lambda: mx.linear(_short(), _short(8, 64)),
    lambda: mx.linear(_short(4, 0), _short(8, 0)),
    lambda: mx.norm(torch.zeros(())),
    lambda: mx.norm(torch.zeros(3, 0)),
    lambda: mx.activation(torch.zeros(())),
    lambda: mx.activation(torch.zeros(3, 0)),
])
def test_what_the_backward_pass_cannot_take_is_refused_in_front(call):
    with pytest.raises(ValueError):
        with torch.no_grad():
            call()


@pytest.mark.parametrize("eps", [-1e-5, float("nan")])
def test_eps_of_norms_is_looked_at_in_front(eps):
    with pytest.raises(ValueError, match="eps"):
        mx.norm(torch.zeros(4, 64), eps=eps)


# ------------------------------------------------------------------------------------------------- negative views

def _negative(t):
    """A view that stands for -t, as the imaginary part of a conjugate does; t's own numbers lie in memory."""
    return torch.complex(torch.zeros_like(t), t).conj().imag


def test_a_column_of_a_conjugate_is_taken_as_what_it_stands_for():
    t = torch.arange(1.0, 6.0).view(5, 1)
    v = _negative(t)
    assert v.is_neg() and v.stride(1) == 2                          # one column: the rows are as good as contiguous
    got = mx._rows(v, "x")
    assert not got.is_neg() and torch.equal(got, -t)
    one = _negative(torch.tensor([3.0]))
    assert one.is_contiguous() and not mx._vector(one).is_neg() and mx._vector(one).item() == -3.0
    assert mx._vector(None) is None
    kept = mx.Packed(torch.zeros(32, dtype=torch.uint8), torch.zeros(16, dtype=torch.uint8), 1, 1)
    out = torch._neg_view(torch.ones(1, 1, dtype=torch.bfloat16))
    for k in (dict(base=out), dict(out=out)):
        with pytest.raises(ValueError, match="contiguous"):
            mx.weight_grad(_short(1, 1), kept, **k)


@gpu
def test_a_negative_column_packed():
    t = torch.arange(1.0, 6.0, device="cuda").view(5, 1)
    assert torch.equal(mx.unpack(mx.pack(_negative(t)), torch.float32), -t)


# ------------------------------------------------------------------------------------------------- under autocast

@gpu
@pytest.mark.parametrize("auto", ["bf16", "f16"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("name", ["layer", "rms", "gelu", "linear", "linear4"])
def test_autocast_changes_nothing(name, dtype, auto):
    """Results and gradients are those without autocast, bit for bit, backward inside it and behind it."""
    d = DT[dtype]
    x, w, dy = numbers(1, 40, 96, d).cuda().requires_grad_(), numbers(2, 64, 96, d).cuda().requires_grad_(), numbers(3, 40, 96 if name in ("layer", "rms", "gelu") else 64, d).cuda()
    nw, b = numbers(4, 1, 96, d)[0].cuda().requires_grad_(), numbers(5, 1, 64, d)[0].cuda().requires_grad_()
    calls = {"layer": (lambda: mx.norm(x, nw), (x, nw)), "rms": (lambda: mx.norm(x, nw, kind="rms"), (x, nw)), "gelu": (lambda: mx.activation(x), (x,)),
             "linear": (lambda: mx.linear(x, w, b), (x, w, b)), "linear4": (lambda: mx.linear(x, w, b, four=True), (x, w, b))}
    call, leaves = calls[name]
    y = call()
    want = [y.detach(), *torch.autograd.grad(y, leaves, dy)]
    for inside in (True, False):
        with torch.autocast("cuda", dtype=DT[auto]):
            y = call()
            assert y.dtype == d
            if inside:
                grads = torch.autograd.grad(y, leaves, dy)
        if not inside:
            grads = torch.autograd.grad(y, leaves, dy)
        assert all(a.dtype == b.dtype and torch.equal(a, b) for a, b in zip([y.detach(), *grads], want))


# ------------------------------------------------------------------------------------------------- nothing is kept where no gradient is taken

@gpu
@pytest.mark.parametrize("name", ["layer", "rms", "gelu", "linear", "linear4"])
def test_nothing_is_kept_for_no_backward_pass(name, monkeypatch):
    d = torch.bfloat16
    x, w, nw = numbers(1, 40, 96, d).cuda(), numbers(2, 64, 96, d).cuda(), numbers(4, 1, 96, d)[0].cuda()
    packs, pack = [], mx.pack
    monkeypatch.setattr(mx, "pack", lambda t, fmt=gb.MX8: packs.append(fmt) or pack(t, fmt))
    call = {"layer": lambda: mx.norm(x, nw), "rms": lambda: mx.norm(x, nw, kind="rms"), "gelu": lambda: mx.activation(x), "linear": lambda: mx.linear(x, w),
            "linear4": lambda: mx.linear(x, w, four=True)}[name]
    four = [gb.MX4] * 2 if name == "linear4" else []
    plain = call()                                                  # no leaf wants a gradient
    assert packs == four and not plain.requires_grad
    for t in (x, w, nw):
        t.requires_grad_()
    for mode in (torch.no_grad, torch.inference_mode):
        del packs[:]
        with mode():
            y = call()
        assert packs == four and torch.equal(y, plain)
    del packs[:]
    y = call()
    assert packs == four + [gb.MX8] and torch.equal(y, plain)
    leaves = [t for t in (x, w, nw) if torch.autograd.grad(y.float().sum(), t, allow_unused=True, retain_graph=True)[0] is not None]
    assert len(leaves) == (1 if name == "gelu" else 2)
    if name.startswith("linear"):                                   # the input's gradient alone reads the weight only
        del packs[:]
        w.requires_grad_(False)
        assert torch.autograd.grad(call().float().sum(), x)[0].shape == x.shape and packs == four


@pytest.mark.parametrize("call", [lambda: mx.norm(torch.ones(4, 64)), lambda: mx.activation(torch.ones(4, 64))])
def test_no_path_on_the_cpu_without_gradients_either(call):
    with pytest.raises(ValueError, match="CUDA"):
        call()


# ------------------------------------------------------------------------------------------------- norms of nearly equal values

@gpu
@pytest.mark.parametrize("cols", [64, 256, 512, 1024, 2048, 4096, 8192, 16384, 32768])
def test_layer_norm_gradients_of_nearly_equal_values(cols):
    """Rows of ones with three values of 15/16, gradients around one: the product sum of gradient and value is a small difference of large sums unless the values are
    taken around a mean.

    The widths are powers of two, so sums, means and deviations are exact in 32 bits, whichever values they are taken around first.  What is left is counted:
    96 half steps (chains of fewer than 64 additions and a handful of operations) of what each term is made of.  A product sum is made of |g| |x - near| and
    |g| |near - mean| for means `near` of parts of the row, whose distances from the row's mean add up to at most those of the values.  The sum of squares, and with it
    r, is off by 96 half steps.
    """
    rng = np.random.default_rng(cols)
    rows = 6
    x = np.ones((rows, cols))
    for row in x:
        row[rng.integers(0, cols, 3)] = 15 / 16
    dy = torch.from_numpy(1 + rng.standard_normal((rows, cols))).float()
    kept, held = packed(torch.from_numpy(x).float(), 8)
    assert (held == x).all()
    g = f64(dy)
    d = x - x.mean(1, keepdims=True)
    r = 1 / np.sqrt((d * d).mean(1, keepdims=True) + 1e-5)
    xn = d * r
    want = r * (g - g.mean(1, keepdims=True) - xn * (g * xn).mean(1, keepdims=True))
    made = r * ((np.abs(g) * np.abs(d)).mean(1, keepdims=True) + 2 * np.abs(g).max(1, keepdims=True) * np.abs(d).mean(1, keepdims=True))
    c = 96 * HALF
    tol = r * (c * (np.abs(g) + np.abs(g).mean(1, keepdims=True)) + np.abs(xn) * (c * made + 3 * c * np.abs((g * xn).mean(1, keepdims=True)))) + c * np.abs(want) + HALF * np.abs(want)
    dx, dw, db = mx.norm_backward(dy.cuda(), kept)
    close(dx, want, tol, "dx")
    close(dw, (g * xn).sum(0), (c + rows * HALF) * np.abs(g * xn).sum(0), "dweight")
    close(db, g.sum(0), rows * HALF * np.abs(g).sum(0), "dbias")
