"""What is timed of the microscaled operators: what a training step does with activations kept in 8 bits and with products in 4 bits.

The search prices strategies by what a layer keeps between its forward and its backward pass and by how fast it multiplies.  The operators
carry two such choices out.  A tensor is held in blocks of 32 along a row with one power of two a block: 8-bit elements (4 exponent and 3
mantissa bits) for what is kept until the backward pass, 4-bit ones (2 and 1) for the operands of a product.

op  "keep"      a tensor is packed and restored: the forward pass keeps it, the backward pass has it back
    "act"       gradient of an activation function whose input was kept in 8 bits
    "norm"      gradients of a layer or root-mean-square norm whose input was kept in 8 bits
    "wgrad"     weight gradient of a linear layer whose input was kept in 8 bits, added to an earlier one where `base` is true
    "product"   product of two tensors held in 4 bits ("packed"), or of a layer's 16- or 32-bit input, packed in the call, with such weights

`pad` is what a row's stride has beyond its length, in elements.  Blocks, codes and scales are laid out as include/galv.h says.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
# (exponent of the largest element's binade, its mantissa): 448 = 1.75 * 2^8, 6 = 1.5 * 2^2
TOP = {8: (8, 1.75), 4: (2, 1.5)}
GRID4 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _case(name, op, rows, cols, dtype, **kw):
    c = {"op": op, "rows": rows, "cols": cols, "dtype": dtype, "fmt": 8, "pad": 0} | kw
    return c if name is None else {"name": name} | c


def listed():
    return [
        # one token's hidden state: the launches are all there is
        _case("keep_one_token", "keep", 1, 2048, "bf16"),
        # what the attention of the heterogeneous stack keeps of two sequences
        _case("keep_sequences", "keep", 8192, 8192, "bf16"),
        # a slice of a wider tensor, rows that end inside a block, 4 bits
        _case("keep_ragged_4bit", "keep", 1537, 5003, "f32", fmt=4, pad=5),
        # the FFN's intermediate activation of one sequence of the heterogeneous stack
        _case("act_ffn", "act", 4096, 32768, "bf16", act="gelu"),
        # a tensor-parallel shard of odd width
        _case("act_ragged", "act", 777, 8191, "f16", act="silu", pad=9),
        # a layer norm of the 175B-shaped decoder, one sequence
        _case("norm_wide", "norm", 2048, 12288, "bf16", kind="layer"),
        # a short tail of a batch, 32-bit gradients
        _case("norm_few_rows", "norm", 33, 2048, "f32", kind="rms"),
        # a projection of the uniform decoder, one sequence
        _case("wgrad_uniform", "wgrad", 2048, 2048, "bf16", n=2048, out="bf16", base=False),
        # the FFN's second matrix of the heterogeneous stack, one sequence, added to the 32-bit gradient of earlier micro-batches
        _case("wgrad_ffn", "wgrad", 4096, 32768, "bf16", n=8192, out="f32", base=True),
        # odd sizes all round
        _case("wgrad_ragged", "wgrad", 1000, 2731, "f16", n=1365, out="f32", base=False, pad=3),
        # a few tokens against a projection of the heterogeneous stack: the weights' bytes are all there is
        _case("product_few_tokens", "product", 7, 8192, "bf16", n=8192, packed=False, bias=True),
        # the FFN's first matrix of the heterogeneous stack, one sequence, input packed in the call
        _case("product_ffn", "product", 4096, 8192, "bf16", n=32768, packed=False, bias=False),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5))))))


def draw(rng):
    op = rng.choice(("keep", "act", "norm", "wgrad", "product"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    pad = rng.choice((0, 0, 0, 8, rng.randint(1, 40)))
    if op in ("wgrad", "product"):
        while True:
            rows, cols, n = _spread(rng, 1, 8192), _spread(rng, 16, 32768), _spread(rng, 16, 32768)
            if rows * cols * n <= 1 << 40 and cols * n <= 1 << 28:
                break
        if op == "wgrad":
            out = rng.choice(("same", "f32"))
            dtype = rng.choice(("bf16", "f16"))
            return _case(None, op, rows, cols, dtype, n=n, out=dtype if out == "same" else out, base=rng.random() < 0.3, pad=pad)
        return _case(None, op, rows, cols, dtype, n=n, packed=rng.random() < 0.4, bias=rng.random() < 0.5, pad=pad)
    while True:
        rows, cols = _spread(rng, 1, 16384), _spread(rng, 16, 16384) if op == "norm" else _spread(rng, 1, 49152)
        if rows * cols <= 1 << 27:
            break
    if op == "keep":
        return _case(None, op, rows, cols, dtype, fmt=rng.choice((8, 8, 4)), pad=pad)
    if op == "act":
        return _case(None, op, rows, cols, dtype, act=rng.choice(("gelu", "gelu_tanh", "silu")), pad=pad)
    return _case(None, op, rows, cols, dtype, kind=rng.choice(("layer", "rms")), pad=pad)


# ------------------------------------------------------------------------------------------------- blocks, in plain operations

def _scale(byte):
    """2^(byte - 127) in 32 bits; NaN for 255."""
    b = byte.to(torch.int32)
    bits = torch.where(b == 0, torch.full_like(b, 0x00400000), b << 23)
    return torch.where(b == 255, torch.full_like(b, 0x7FC00000), bits).view(torch.float32)


def _blocks(x):
    """[rows, blocks, 32] of a matrix in 32 bits, zeros behind a row's end."""
    rows, cols = x.shape
    nb = -(-cols // 32)
    p = torch.zeros(rows, nb * 32, dtype=torch.float32, device=x.device)
    p[:, :cols] = x
    return p.view(rows, nb, 32)


def _quantise(x, fmt):
    """(elements as 32-bit values [rows, blocks, 32], exponent bytes [rows, blocks]): the smallest power of two under which no element of
    the block passes the largest value of the format, then to nearest, ties to even."""
    b = _blocks(x)
    amax = b.abs().amax(2)
    m, e = torch.frexp(amax)                                            # amax = m * 2^e, m in [1/2, 1)
    top, mant = TOP[fmt]
    s = e.to(torch.int32) - 1 - top + (2 * m > mant).to(torch.int32)
    byte = torch.where(amax == 0, torch.zeros_like(s), (s + 127).clamp(0, 254))
    v = b * ((254 - byte) << 23).view(torch.float32)[:, :, None]
    if fmt == 8:
        q = v.to(torch.float8_e4m3fn).to(torch.float32)
    else:
        a = v.abs()
        step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
        q = torch.copysign(torch.round(a / step) * step, v)
    return q, byte


def _restore(q, byte, cols):
    rows = q.shape[0]
    return (q * _scale(byte)[:, :, None]).reshape(rows, -1)[:, :cols]


def _rounded(v, dtype):
    """To the type a caller asked for; what was kept as a number stays one."""
    return v.clamp(-65504.0, 65504.0).to(dtype) if dtype == torch.float16 else v.to(dtype)


def _lay_scales(byte, fmt):
    rows, nb = byte.shape
    if fmt == 8:                                                        # [rows][blocks up to a multiple of 16]
        out = torch.zeros(rows, -(-nb // 16) * 16, dtype=torch.uint8, device=byte.device)
        out[:, :nb] = byte.to(torch.uint8)
        return out.reshape(-1)
    r128, nb4 = -(-rows // 128), -(-nb // 4)                            # tiles of 128 rows x 4 blocks: [32 rows][4 groups of rows][4 blocks]
    out = torch.zeros(r128 * 128, nb4 * 4, dtype=torch.uint8, device=byte.device)
    out[:rows, :nb] = byte.to(torch.uint8)
    return out.view(r128, 4, 32, nb4, 4).permute(0, 3, 2, 1, 4).contiguous().view(-1)


def _read_scales(scales, rows, cols, fmt):
    nb = -(-cols // 32)
    if fmt == 8:
        return scales.view(rows, -1)[:, :nb]
    r128, nb4 = -(-rows // 128), -(-nb // 4)
    return scales.view(r128, nb4, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(r128 * 128, nb4 * 4)[:rows, :nb]


def _codes(q, fmt):
    rows = q.shape[0]
    if fmt == 8:
        return q.to(torch.float8_e4m3fn).view(torch.uint8).reshape(-1)
    grid = torch.tensor(GRID4, device=q.device)
    c = torch.searchsorted(grid, q.abs()).to(torch.uint8) | (torch.signbit(q).to(torch.uint8) << 3)
    c = c.view(rows, -1)
    return (c[:, 0::2] | (c[:, 1::2] << 4)).reshape(-1)


def _pack(x, fmt):
    q, byte = _quantise(x, fmt)
    return {"codes": _codes(q, fmt), "scales": _lay_scales(byte, fmt), "rows": x.shape[0], "cols": x.shape[1], "fmt": fmt}


def _unpack(p):
    """The kept values in 32 bits."""
    rows, cols, fmt = p["rows"], p["cols"], p["fmt"]
    nb = -(-cols // 32)
    if fmt == 8:
        q = p["codes"].view(torch.float8_e4m3fn).to(torch.float32).view(rows, nb, 32)
    else:
        c = p["codes"].view(rows, nb, 16)
        c = torch.stack((c & 15, c >> 4), 3).view(rows, nb, 32).to(torch.int64)
        table = torch.tensor(GRID4 + tuple(-g for g in GRID4), device=c.device)
        q = table[c]
    return _restore(q, _read_scales(p["scales"], rows, cols, fmt), cols)


# ------------------------------------------------------------------------------------------------- inputs

def _activations(g, rows, cols, dtype, pad=0):
    """Hidden states: normal, a few channels some twenty times as large, rows of different size."""
    dev = g.device
    x = torch.randn(rows, cols, generator=g, device=dev)
    x *= 0.5 + torch.rand(rows, 1, generator=g, device=dev)
    x *= torch.where(torch.rand(cols, generator=g, device=dev) < 0.004, 20.0, 1.0)
    return _strided(x, dtype, pad)


def _strided(x, dtype, pad):
    if not pad:
        return x.to(dtype)
    wide = torch.zeros(x.shape[0], x.shape[1] + pad, dtype=dtype, device=x.device)
    wide[:, :x.shape[1]] = x.to(dtype)
    return wide[:, :x.shape[1]]


def _gradients(g, rows, cols, dtype, pad=0):
    return _strided(torch.randn(rows, cols, generator=g, device=g.device) * 0.02, dtype, pad)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rows, cols, dt, pad = case["rows"], case["cols"], DTYPES[case["dtype"]], case["pad"]
    s = {"case": case}
    if case["op"] == "keep":
        s["x"] = _activations(g, rows, cols, dt, pad)
        return s
    if case["op"] == "product":
        x = _activations(g, rows, cols, dt, pad)
        s["x"] = _pack(x, 4) if case["packed"] else x
        s["w"] = _pack(torch.randn(case["n"], cols, generator=g, device="cuda") * cols ** -0.5, 4)
        s["bias"] = (torch.randn(case["n"], generator=g, device="cuda") * 0.1).to(dt) if case["bias"] else None
        return s
    s["kept"] = _pack(_activations(g, rows, cols, torch.bfloat16 if case["op"] == "wgrad" else dt), 8)
    if case["op"] == "wgrad":
        s["dy"] = _gradients(g, rows, case["n"], dt, pad)
        s["base"] = torch.randn(case["n"], cols, generator=g, device="cuda").mul_(0.05).to(DTYPES[case["out"]]) if case["base"] else None
        return s
    s["dy"] = _gradients(g, rows, cols, dt, pad)
    if case["op"] == "norm":
        s["weight"] = (1 + 0.1 * torch.randn(cols, generator=g, device="cuda")).to(dt)
    return s


# ------------------------------------------------------------------------------------------------- one pass

EPS = 1e-5


def _plain(s):
    c = s["case"]
    dt = DTYPES[c["dtype"]]
    if c["op"] == "keep":
        q, byte = _quantise(s["x"], c["fmt"])
        return _rounded(_restore(q, byte, c["cols"]), dt)
    if c["op"] == "product":
        if c["packed"]:
            a = _unpack(s["x"])
        else:
            q, byte = _quantise(s["x"], 4)
            a = _restore(q, byte, c["cols"])
        y = a @ _unpack(s["w"]).t()
        if s["bias"] is not None:
            y = y + s["bias"].float()
        return y.to(dt)
    x, dy = _unpack(s["kept"]), s["dy"].float()
    if c["op"] == "wgrad":
        x = _rounded(x, dt).float()                                     # the product takes both operands in the gradient's type
        dw = dy.t() @ x
        if s["base"] is not None:
            dw = s["base"].float() + dw
        return dw.to(DTYPES[c["out"]])
    if c["op"] == "act":
        if c["act"] == "gelu":
            d = 0.5 * (1 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(-0.5 * x * x) * (1 / math.sqrt(2 * math.pi))
        elif c["act"] == "gelu_tanh":
            k = math.sqrt(2 / math.pi)
            t = torch.tanh(k * (x + 0.044715 * x ** 3))
            d = 0.5 * (1 + t) + 0.5 * x * (1 - t * t) * k * (1 + 3 * 0.044715 * x * x)
        else:
            sg = 1 / (1 + torch.exp(-x))
            d = sg * (1 + x * (1 - sg))
        return (dy * d).to(dt)
    layer = c["kind"] == "layer"
    if layer:
        x = x - x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt((x * x).mean(1, keepdim=True) + EPS)
    xn = x * rstd
    gy = dy * s["weight"].float()
    dx = gy - xn * (gy * xn).mean(1, keepdim=True)
    if layer:
        dx = dx - gy.mean(1, keepdim=True)
    out = {"dx": (dx * rstd).to(dt), "dweight": (dy * xn).sum(0)}
    if layer:
        out["dbias"] = dy.sum(0)
    return out


def _packed(p):
    from paper_2504_03662_b200 import mx
    return mx.Packed(p["codes"], p["scales"], p["rows"], p["cols"], p["fmt"])


def _own(s):
    from paper_2504_03662_b200 import mx
    c = s["case"]
    dt = DTYPES[c["dtype"]]
    if c["op"] == "keep":
        return mx.unpack(mx.pack(s["x"], c["fmt"]), dt)
    if c["op"] == "product":
        a = _packed(s["x"]) if c["packed"] else mx.pack(s["x"], 4)
        return mx.matmul(a, _packed(s["w"]), dt, bias=s["bias"])
    kept = _packed(s["kept"])
    if c["op"] == "wgrad":
        return mx.weight_grad(s["dy"], kept, DTYPES[c["out"]], base=s["base"])
    if c["op"] == "act":
        return mx.act_backward(s["dy"], kept, c["act"])
    dx, dweight, dbias = mx.norm_backward(s["dy"], kept, s["weight"], c["kind"], EPS)
    return {"dx": dx, "dweight": dweight} if c["kind"] == "rms" else {"dx": dx, "dweight": dweight, "dbias": dbias}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------- work, and the definition in 64 bits

def _held(rows, cols, fmt):
    nb = -(-cols // 32)
    return rows * nb * (32 * fmt // 8 + 1)


def work(case):
    rows, cols = case["rows"], case["cols"]
    el = DTYPES[case["dtype"]].itemsize
    if case["op"] == "keep":                                            # packed, then restored: what is held is written and read
        return {"bytes": 2 * rows * cols * el + 2 * _held(rows, cols, case["fmt"]), "flops": 4 * rows * cols}
    if case["op"] == "act":
        return {"bytes": 2 * rows * cols * el + _held(rows, cols, 8), "flops": 20 * rows * cols}
    if case["op"] == "norm":
        return {"bytes": 2 * rows * cols * el + _held(rows, cols, 8) + cols * (el + 8), "flops": 16 * rows * cols}
    n = case["n"]
    if case["op"] == "wgrad":
        out = DTYPES[case["out"]].itemsize
        return {"bytes": rows * n * el + _held(rows, cols, 8) + n * cols * out * (2 if case["base"] else 1), "flops": 2 * rows * n * cols}
    a = _held(rows, cols, 4) if case["packed"] else rows * cols * el
    return {"bytes": a + _held(n, cols, 4) + rows * n * el + (n * el if case["bias"] else 0), "flops": 2 * rows * n * cols}


def _two_to(k):
    """2^k in 64 bits, exactly."""
    return ((k.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_values(p):
    """What codes and scales stand for, from their bits."""
    rows, cols, fmt = p["rows"], p["cols"], p["fmt"]
    nb = (cols + 31) // 32
    c = p["codes"].long().view(rows, nb, -1)
    if fmt == 4:
        c = torch.cat((c.unsqueeze(3) & 15, c.unsqueeze(3) >> 4), 3).flatten(2)
        sign, e, m = c >> 3, (c >> 1) & 3, c & 1
        mag = torch.where(e == 0, m * 0.5, (1 + m * 0.5) * _two_to(e - 1))
    else:
        sign, e, m = c >> 7, (c >> 3) & 15, c & 7
        mag = torch.where(e == 0, m.double() * 2.0 ** -9, (8 + m).double() * _two_to(e - 10))
    v = torch.where(sign == 1, -mag.double(), mag.double())
    r = torch.arange(rows, device=c.device)[:, None]
    b = torch.arange(nb, device=c.device)[None, :]
    at = r * (-(-nb // 16) * 16) + b if fmt == 8 else ((r // 128) * (-(-nb // 4)) + b // 4) * 512 + (r % 32) * 16 + (r // 32 % 4) * 4 + b % 4
    return (v * _two_to(p["scales"][at].long() - 127)[:, :, None]).flatten(1)[:, :cols]


def _exact_kept(x, fmt):
    """The values that a matrix is held as: nearest multiples of each element's quantum, which is the format's under the block's power of two."""
    rows, cols = x.shape
    nb = (cols + 31) // 32
    b = torch.nn.functional.pad(x.double(), (0, nb * 32 - cols)).view(rows, nb, 32)
    most, least, bits = (448.0, -6.0, 3) if fmt == 8 else (6.0, 0.0, 1)
    lim = b.abs().amax(2, keepdim=True) / most
    k = torch.ceil(torch.log2(lim.clamp(min=2.0 ** -300)))
    k = torch.where(_two_to(k - 1) >= lim, k - 1, torch.where(_two_to(k) < lim, k + 1, k))
    unit = _two_to(torch.where(lim == 0, torch.zeros_like(k), k.clamp(min=-127.0)))
    v = b / unit
    e = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** (least - 1))))
    e = torch.where(_two_to(e) > v.abs(), e - 1, torch.where(_two_to(e + 1) <= v.abs(), e + 1, e)).clamp(min=least)
    quantum = _two_to(e - bits)
    return (torch.round(v / quantum) * quantum * unit).flatten(1)[:, :cols]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "keep":
        return _exact_kept(s["x"], case["fmt"])
    if op == "product":
        a = _exact_values(s["x"]) if case["packed"] else _exact_kept(s["x"], 4)
        y = torch.matmul(a, _exact_values(s["w"]).transpose(0, 1))
        return y if s["bias"] is None else y + s["bias"].double()
    x, dy = _exact_values(s["kept"]), s["dy"].double()
    if op == "wgrad":
        dw = torch.matmul(dy.transpose(0, 1), x)
        return dw if s["base"] is None else dw + s["base"].double()
    if op == "act":
        x.requires_grad_(True)
        with torch.enable_grad():
            if case["act"] == "silu":
                y = x * torch.sigmoid(x)
            elif case["act"] == "gelu":
                y = x * 0.5 * torch.erfc(-x / 2 ** 0.5)
            else:
                y = 0.5 * x * (1 + torch.tanh((2 / math.pi) ** 0.5 * (x + 0.044715 * x * x * x)))
            return torch.autograd.grad(y, x, dy)[0]
    x.requires_grad_(True)
    w = s["weight"].double().requires_grad_(True)
    with torch.enable_grad():
        if case["kind"] == "layer":
            bias = torch.zeros_like(w).requires_grad_(True)
            var, mean = torch.var_mean(x, 1, unbiased=False, keepdim=True)
            y = (x - mean) / torch.sqrt(var + EPS) * w + bias
            dx, dw, db = torch.autograd.grad(y, (x, w, bias), dy)
            return {"dx": dx, "dweight": dw, "dbias": db}
        y = x / torch.sqrt(torch.mean(x * x, 1, keepdim=True) + EPS) * w
        dx, dw = torch.autograd.grad(y, (x, w), dy)
    return {"dx": dx, "dweight": dw}
