"""What is timed of the products in 8-bit integers and of the experts' products.

An 8-bit matrix has one scale a row, s = max(largest magnitude, 2^-100) / 127, and whole numbers, the nearest to x / s: rows are tokens on one
side of a product and output channels on the other.  Experts' products take rows sorted by expert: `ends[e]` is where expert e's rows end, rows behind the
last end belong to none and give zeros.

op  "i8"        a layer's input is put into 8-bit integers and multiplied by weights held so: y = (qx qw^T) * sx * sw + bias
    "experts"   each row by its expert's weights, in 16 bits ("forward") or in 8-bit integers ("i8", input packed in the call)
    "step"      forward and backward pass of the same as a training step makes them: y, dx, dw and db where there is a bias
    "wgrad"     weight gradient of experts, added to an earlier one where `base` is true

`pad` is what a row's stride has beyond its length, in elements; `behind` how many rows lie behind the last end; `skew` how unevenly experts are chosen.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _case(name, op, rows, cols, n, dtype, **kw):
    c = {"op": op, "rows": rows, "cols": cols, "n": n, "dtype": dtype, "pad": 0, "bias": False}
    if op != "i8":
        c |= {"experts": 8, "skew": 0.5, "behind": 0}
    c |= kw
    return c if name is None else {"name": name} | c


def listed():
    return [
        # one token against a projection of the heterogeneous stack: the weights' bytes are all there is
        _case("i8_one_token", "i8", 1, 8192, 8192, "bf16", bias=True),
        # a batch of decoding sequences, the uniform decoder's FFN
        _case("i8_few_tokens", "i8", 48, 2048, 8192, "f16"),
        # the FFN's first matrix of the heterogeneous stack, one sequence
        _case("i8_ffn", "i8", 4096, 8192, 32768, "bf16"),
        # odd sizes all round, a slice of a wider tensor, 32-bit numbers in and out
        _case("i8_ragged", "i8", 777, 5003, 2731, "f32", pad=5, bias=True),
        # one token that two of sixteen experts share
        _case("experts_one_token", "experts", 2, 2048, 8192, "bf16", form="forward", experts=16),
        # four sequences of the uniform decoder, every token by two of eight experts
        _case("experts_forward", "experts", 16384, 2048, 8192, "bf16", form="forward"),
        # a batch of decoding sequences over many experts, most of which get one token or none
        _case("experts_i8_decode", "experts", 64, 2048, 4096, "bf16", form="i8", experts=64, skew=1.0),
        # a long prompt over narrow experts of the heterogeneous stack, in a padded batch
        _case("experts_i8_prompt", "experts", 8192, 8192, 2048, "bf16", form="i8", experts=16, behind=192),
        # a training step of two sequences, every token by two of sixteen experts
        _case("step_uniform", "step", 8192, 2048, 4096, "bf16", experts=16),
        # odd sizes, an expert without rows, a bias, rows behind the last end
        _case("step_ragged", "step", 777, 1365, 2731, "f16", experts=7, skew=1.5, behind=21, bias=True, pad=3),
        # the experts' second matrix, added to the 32-bit gradient of earlier micro-batches
        _case("wgrad_onto_base", "wgrad", 16384, 8192, 2048, "bf16", out="f32", base=True),
        # a micro-batch's few rows an expert: writing the gradient is all there is
        _case("wgrad_few_rows", "wgrad", 300, 2048, 1365, "f16", out="f16", base=False, experts=24, skew=1.0, behind=4),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5))))))


def draw(rng):
    op = rng.choice(("i8", "experts", "step", "wgrad"))
    pad = rng.choice((0, 0, 0, 8, rng.randint(1, 40)))
    bias = rng.random() < 0.4
    if op == "i8":
        while True:
            rows, cols, n = _spread(rng, 1, 8192), _spread(rng, 16, 32768), _spread(rng, 16, 32768)
            if rows * cols * n <= 1 << 39 and cols * n <= 1 << 28:
                break
        return _case(None, op, rows, cols, n, rng.choice(("bf16", "bf16", "f16", "f32")), pad=pad, bias=bias)
    while True:
        rows, cols, n, e = _spread(rng, 1, 16384), _spread(rng, 16, 8192), _spread(rng, 16, 8192), _spread(rng, 1, 128)
        if rows * cols * n <= (1 << 38 if op == "experts" else 1 << 36) and e * cols * n <= 1 << 28:
            break
    kw = {"experts": e, "skew": rng.choice((0.0, 0.5, 1.0, 2.0)), "behind": rng.choice((0, 0, rng.randint(0, rows // 2))), "pad": pad}
    dtype = rng.choice(("bf16", "bf16", "f16"))
    if op == "experts":
        return _case(None, op, rows, cols, n, dtype, form=rng.choice(("forward", "i8")), bias=bias, **kw)
    if op == "step":
        return _case(None, op, rows, cols, n, dtype, bias=bias, **kw)
    return _case(None, op, rows, cols, n, dtype, out=rng.choice((dtype, "f32")), base=rng.random() < 0.4, **kw)


# ------------------------------------------------------------------------------------------------- inputs

def _strided(x, dtype, pad):
    if not pad:
        return x.to(dtype)
    wide = torch.zeros(x.shape[0], x.shape[1] + pad, dtype=dtype, device=x.device)
    wide[:, :x.shape[1]] = x.to(dtype)
    return wide[:, :x.shape[1]]


def _activations(g, rows, cols, dtype, pad=0):
    """Hidden states: normal, a few channels some twenty times as large, rows of different size."""
    x = torch.randn(rows, cols, generator=g, device="cuda")
    x *= 0.5 + torch.rand(rows, 1, generator=g, device="cuda")
    x *= torch.where(torch.rand(cols, generator=g, device="cuda") < 0.004, 20.0, 1.0)
    return _strided(x, dtype, pad)


def _scales(x):
    """One scale a row, a number of 32 bits."""
    return (x.abs().amax(1).double().clamp(min=2.0 ** -100) / 127).float()


def _whole(x, scale):
    """The nearest whole numbers to x / scale; 64 bits, so that a quotient next to a half stays on its side."""
    return torch.round(x.double() / scale.double()[:, None])


def _held(x):
    """A matrix in 8-bit integers as a program keeps it: rows up to a multiple of 16 bytes with zeros behind their ends, and the scales."""
    rows, cols = x.shape
    scales = _scales(x)
    codes = torch.zeros(rows, -(-cols // 16) * 16, dtype=torch.int8, device=x.device)
    codes[:, :cols] = _whole(x, scales).to(torch.int8)
    return {"codes": codes, "scales": scales, "rows": rows, "cols": cols}


def _counts(case, seed):
    """Rows of each expert, as a router gives them."""
    r = np.random.default_rng(seed)
    p = np.exp(case["skew"] * r.standard_normal(case["experts"]))
    return r.multinomial(case["rows"] - case["behind"], p / p.sum()).tolist()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rows, cols, n, dt = case["rows"], case["cols"], case["n"], DTYPES[case["dtype"]]
    s = {"case": case, "x": _activations(g, rows, cols, dt, case["pad"])}
    e = 1
    if case["op"] != "i8":
        e = case["experts"]
        s["counts"] = _counts(case, seed)
        s["ends"] = torch.tensor(s["counts"], dtype=torch.int64).cumsum(0).to(torch.int32).cuda()
    s["bias"] = (torch.randn(e, n, generator=g, device="cuda") * 0.1).to(dt) if case["bias"] else None
    if case["op"] in ("step", "wgrad"):
        s["dy"] = (torch.randn(rows, n, generator=g, device="cuda") * 0.02).to(dt)
    if case["op"] == "wgrad":
        s["base"] = torch.randn(e, n, cols, generator=g, device="cuda").mul_(0.05).to(DTYPES[case["out"]]) if case["base"] else None
        return s
    w = torch.randn(e, n, cols, generator=g, device="cuda") * cols ** -0.5
    if case["op"] == "i8" or case.get("form") == "i8":
        s["w"] = _held(w.view(e * n, cols))
    else:
        s["w"] = w.to(dt)
    if case["op"] == "i8" and case["bias"]:
        s["bias"] = s["bias"][0]
    if case["op"] == "step":
        s["leaves"] = [t for t in (s["x"], s["w"], s["bias"]) if t is not None]
        for t in s["leaves"]:
            t.requires_grad_(True)
    return s


# ------------------------------------------------------------------------------------------------- one pass

def _by_expert(counts, f, rows=None):
    """f(expert, first row, last row) for the experts in turn; of `rows` rows, those behind the last end are zeros."""
    out, at = [], 0
    for e, count in enumerate(counts):
        if count or rows is None:
            out.append(f(e, at, at + count))
        at += count
    if rows is None:
        return torch.stack(out)
    like = out[0] if out else f(0, 0, 0)
    return torch.cat(out + [torch.zeros(rows - at, like.shape[1], dtype=like.dtype, device=like.device)])


def _plain(s):
    c = s["case"]
    dt, rows, n, cols = DTYPES[c["dtype"]], c["rows"], c["n"], c["cols"]
    with torch.no_grad():
        bias = None if s["bias"] is None else s["bias"].float()
        if c["op"] == "i8" or c.get("form") == "i8":
            scale = _scales(s["x"])
            q = _whole(s["x"], scale).float()
            w, ws = s["w"]["codes"][:, :cols], s["w"]["scales"]
            if c["op"] == "i8":
                y = q @ w.float().t() * scale[:, None] * ws
                return (y if bias is None else y + bias).to(dt)
            w, ws = w.unflatten(0, (-1, n)), ws.view(-1, n)

            def one(e, a, b):
                y = q[a:b] @ w[e].float().t() * scale[a:b, None] * ws[e]
                return y if bias is None else y + bias[e]
            return _by_expert(s["counts"], one, rows).to(dt)
        x = s["x"].float()
        if c["op"] == "wgrad":
            dy = s["dy"].float()
            dw = _by_expert(s["counts"], lambda e, a, b: dy[a:b].t() @ x[a:b])
            return (dw if s["base"] is None else s["base"].float() + dw).to(DTYPES[c["out"]])
        w = s["w"]

        def forward(e, a, b):
            y = x[a:b] @ w[e].float().t()
            return y if bias is None else y + bias[e]
        y = _by_expert(s["counts"], forward, rows).to(dt)
        if c["op"] == "experts":
            return y
        dy = s["dy"].float()
        out = {"y": y, "dx": _by_expert(s["counts"], lambda e, a, b: dy[a:b] @ w[e].float(), rows).to(dt),
               "dw": _by_expert(s["counts"], lambda e, a, b: dy[a:b].t() @ x[a:b]).to(dt)}
        if bias is not None:
            out["db"] = _by_expert(s["counts"], lambda e, a, b: dy[a:b].sum(0)).to(dt)
        return out


def _own(s):
    from paper_2504_03662_b200 import experts, i8
    c = s["case"]
    if c["op"] == "i8" or c.get("form") == "i8":
        w = i8.Packed(s["w"]["codes"], s["w"]["scales"], s["w"]["rows"], s["w"]["cols"])
        return i8.linear(s["x"], w, s["bias"]) if c["op"] == "i8" else experts.matmul(s["x"], w, s["ends"], s["bias"])
    if c["op"] == "wgrad":
        return experts.weight_grad(s["dy"], s["x"], s["ends"], DTYPES[c["out"]], base=s["base"])
    if c["op"] == "experts":
        return experts.matmul(s["x"], s["w"], s["ends"], s["bias"])
    y = experts.linear(s["x"], s["w"], s["ends"], s["bias"])
    grads = torch.autograd.grad(y, s["leaves"], s["dy"])
    return {"y": y.detach()} | dict(zip(("dx", "dw", "db"), grads))


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------- work, and the definition in 64 bits

def work(case):
    rows, cols, n = case["rows"], case["cols"], case["n"]
    el = DTYPES[case["dtype"]].itemsize
    flops = 2 * rows * cols * n
    if case["op"] == "i8":
        return {"bytes": rows * (cols + n) * el + n * (cols + 4) + (n * el if case["bias"] else 0), "flops": flops}
    rows -= case["behind"]
    most = sum(int(np.count_nonzero(_counts(case, k))) for k in range(8)) / 8   # experts that have rows, as a rule: their weights are read
    flops = 2 * rows * cols * n
    if case["op"] == "wgrad":
        out = DTYPES[case["out"]].itemsize
        return {"bytes": rows * (cols + n) * el + case["experts"] * n * cols * out * (2 if case["base"] else 1), "flops": flops}
    moved = rows * cols * el + case["rows"] * n * el + (most * n * el if case["bias"] else 0)
    if case["op"] == "experts":
        return {"bytes": moved + most * n * (cols + 4 if case["form"] == "i8" else cols * el), "flops": flops}
    # forward, then dx and dw: x, w and dy are each read by two of the three products, which lie a whole pass apart for x and w
    moved += rows * n * el + case["rows"] * cols * el + rows * cols * el + 2 * most * n * cols * el + case["experts"] * n * cols * el
    return {"bytes": moved, "flops": 3 * flops}


def _exact_held(x):
    """The numbers that rows in 8-bit integers stand for, as whole numbers and scales in 64 bits."""
    x = x.detach().double()
    top = torch.maximum(x.max(1, keepdim=True).values, -x.min(1, keepdim=True).values)
    scale = (torch.clamp(top, min=2.0 ** -100) / 127).to(torch.float32).double()
    low = torch.floor(x / scale)
    up = x - low * scale
    half = scale / 2
    odd = torch.remainder(low, 2) == 1
    return low + ((up > half) | ((up == half) & odd)).double(), scale


def exact(case, seed):
    s = prepare(case, seed)
    rows, cols, n = case["rows"], case["cols"], case["n"]
    bias = None if s["bias"] is None else s["bias"].detach().double()
    if case["op"] == "i8" or case.get("form") == "i8":
        q, scale = _exact_held(s["x"])
        x = q * scale
        w = s["w"]["codes"][:, :cols].double() * s["w"]["scales"].double().unsqueeze(1)
    else:
        x, w = s["x"].detach().double(), s["w"].detach().double() if "w" in s else None
    if case["op"] == "i8":
        y = torch.matmul(x, w.transpose(0, 1))
        return y if bias is None else y + bias
    bounds = [0] + torch.cumsum(torch.tensor(s["counts"]), 0).tolist()
    e = case["experts"]
    if case["op"] == "wgrad":
        dw = torch.zeros(e, n, cols, dtype=torch.float64, device="cuda") if s["base"] is None else s["base"].double()
        for i in range(e):
            dw[i] += torch.einsum("tn,tk->nk", s["dy"][bounds[i]:bounds[i + 1]].double(), x[bounds[i]:bounds[i + 1]])
        return dw
    w = w.reshape(e, n, cols)
    y = torch.zeros(rows, n, dtype=torch.float64, device="cuda")
    for i in range(e):
        at = slice(bounds[i], bounds[i + 1])
        y[at] = torch.einsum("tk,nk->tn", x[at], w[i])
        if bias is not None:
            y[at] += bias[i]
    if case["op"] == "experts":
        return y
    dy = s["dy"].double()
    dx, dw, db = torch.zeros_like(x), torch.zeros_like(w), torch.zeros(e, n, dtype=torch.float64, device="cuda")
    for i in range(e):
        at = slice(bounds[i], bounds[i + 1])
        dx[at] = torch.einsum("tn,nk->tk", dy[at], w[i])
        dw[i] = torch.einsum("tn,tk->nk", dy[at], x[at])
        db[i] = torch.sum(dy[at], 0)
    out = {"y": y, "dx": dx, "dw": dw}
    if bias is not None:
        out["db"] = db
    return out
