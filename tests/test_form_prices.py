"""What strategies in 8 and 4 bits cost, against bytes and seconds counted from the tensors that they stand for."""
import numpy as np
import pytest

from paper_2504_03662_b200 import inputs

gpu = pytest.mark.gpu


def one_layer(ckpt, sp, bytes_per_elem):
    """One layer of 2048 tokens x 1024 on two tensor-parallel GPUs, which keeps three matrices of that size (one whole, two shared out) and no masks; with
    checkpointing its input."""
    layers = np.zeros((1, 1), inputs.LAYER_DESC)
    for k, v in dict(h=1024.0, seq=1024.0, heads=8.0, c_lin=24.0, p_coef=12.0, act_rep=2.0, act_tp=4.0).items():
        layers[k] = v
    strat = np.array([(2, 4, 3, ckpt, sp, 0, 1.0)], inputs.STRATEGY_DESC)
    inst = np.zeros(1, inputs.INST_PARAMS)
    for k, v in dict(b=2.0, act_mult=3.0, flops_rate=1e15, bw_tp=4e11, bw_dp=4e11, bytes_per_elem=bytes_per_elem, bin_bytes=64.0, time_unit_ns=1.0).items():
        inst[k] = v
    return inputs.Workload("one_layer", 1, 1, 1, 1000, np.ones(1, np.int32), layers=layers, strat=strat, inst=inst)


@gpu
@pytest.mark.parametrize("bytes_per_elem", [1.0, 2.0, 4.0])
@pytest.mark.parametrize("ckpt,sp", [(0, 0), (0, 1), (1, 0), (1, 1)])
def test_kept_bytes_are_those_of_the_tensors(ckpt, sp, bytes_per_elem):
    from paper_2504_03662_b200 import binding as gb, mx
    from paper_2504_03662_b200.search import SearchBuffers
    galv = gb.Galv(0)
    w = one_layer(ckpt, sp, bytes_per_elem).with_forms([(8, 0, 0.0, 1.0)])
    sb = SearchBuffers(galv, w)
    sb.eval_costs()
    tokens, h = 2048, 1024
    whole, shared = (1, 0) if ckpt else (1, 2)
    sizes = [(tokens // 2 if sp else tokens, h)] * whole + [(tokens, h // 2)] * shared
    plain = sum(2 * r * c for r, c in sizes)                        # the cost model's activations are 16-bit numbers
    held = sum(mx.codes_bytes(r, c) + mx.scales_bytes(r, c) for r, c in sizes)
    mem = sb.mem_bytes.cpu().numpy()[0, 0]
    assert mem[0] == mem[1] == 12 * h * h / 2 * 16 / 4 + 3 * plain
    assert sb.mem_q.cpu().numpy()[0, 0].tolist() == [mem[0] / 64, (mem[0] - 3 * (plain - held)) / 64]
    galv.close()


@pytest.fixture
def priced_calls(monkeypatch):
    """Prices for measure_forms: a call that it times costs 1 second and what `cost` says for each microscaled operator in it.  Returns (cost, what each
    timed call ran, a list that every operator is written to)."""
    from paper_2504_03662_b200 import mx, search
    cost, timed, ran = {}, [], []

    def counting(name):
        f = getattr(mx, name)

        def call(*a, **k):
            ran.append(f"{name}{a[1]}" if name == "pack" and len(a) > 1 else name)
            return f(*a, **k)
        return call

    for name in ("pack", "unpack", "act_backward", "norm_backward", "weight_grad", "matmul"):
        monkeypatch.setattr(mx, name, counting(name))

    def seconds(f, reps=5):
        del ran[:]
        f()
        timed.append(list(ran))
        return 1.0 + sum(cost.get(op, 0.0) for op in ran)

    monkeypatch.setattr(search, "_seconds", seconds)
    return cost, timed, ran


@gpu
def test_the_speed_of_products_is_that_of_the_layer_that_carries_them_out(priced_calls):
    """What is timed in 4 bits packs and multiplies what mx.linear does."""
    import torch
    from paper_2504_03662_b200 import binding as gb, mx
    from paper_2504_03662_b200.search import measure_forms
    cost, timed, ran = priced_calls
    cost.update({"pack4": 4.0, "matmul": 3.0})
    galv = gb.Galv(0)
    form = measure_forms(galv, 64, 128, keep=False)
    del ran[:]
    mx.linear(torch.ones(128, 64, device="cuda", dtype=torch.bfloat16), torch.ones(64, 64, device="cuda", dtype=torch.bfloat16), four=True)
    assert sorted(ran) == ["matmul", "pack4", "pack4"] and sorted(timed[-1]) == sorted(ran)
    assert form["mul_speed"].tolist() == [1.0 / 12.0]
    galv.close()


@gpu
@pytest.mark.parametrize("dearest,price", [("weight_grad", 100.0), ("norm_backward", 100.0), ("act_backward", 100.0), ("unpack", 101.0), (None, 1.0)])
def test_keeping_in_8_bits_costs_packing_and_its_dearest_use(priced_calls, dearest, price):
    """Each use costs what it takes longer than the plain backward pass; restoring has none beside it (and is the dearest where all are alike)."""
    from paper_2504_03662_b200 import binding as gb
    from paper_2504_03662_b200.search import measure_forms
    cost, timed, ran = priced_calls
    cost.update({"pack": 6.0, dearest: 100.0})
    galv = gb.Galv(0)
    form = measure_forms(galv, 64, 128, multiply=False)
    assert form["keep_s_per_byte"].tolist() == [(7.0 + price) / (128 * 64 * 2)]
    galv.close()


def test_forms_of_forms_are_refused():
    """A second round would have dropped the first one's forms and kept its strategies."""
    w = inputs.config1().with_forms([(8, 0, 1e-12, 1.0)])
    with pytest.raises(ValueError, match="already"):
        w.with_forms([(0, 4, 0.0, 2.0)])


@pytest.mark.parametrize("hidden,tokens", [(1024, 0), (0, 16), (-1, 16)])
def test_rates_of_nothing_are_refused(hidden, tokens):
    """Seconds for each of no bytes: a division by zero in the middle of the measurement before."""
    from types import SimpleNamespace
    from paper_2504_03662_b200.search import measure_forms
    with pytest.raises(ValueError, match="at least 1"):
        measure_forms(SimpleNamespace(device=0), hidden, tokens)


def test_workloads_are_made_as_they_were_before_they_had_forms():
    w = inputs.config1()
    again = inputs.Workload(w.name, w.B, w.Lmax, w.S, w.M, w.L, None, None, None, w.layers, w.strat, w.inst, {"pp": 1})
    assert again.meta == {"pp": 1} and again.forms is None
    f = w.with_forms([(8, 0, 1e-12, 1.0)])
    assert f.take(slice(0, 2)).forms is f.forms and f.take(slice(0, 2)).meta == f.meta


def test_masks_are_a_part_of_the_layers():
    w = inputs.config3(4)
    held = w.with_forms([(8, 0, 1e-12, 1.0)], masks=1.0)
    assert (held.form_layers["act_rep"] == 4.0).all() and (held.layers["act_rep"] == 5.0).all() and (held.take(slice(1, 3)).masks == 1.0).all()
    each = np.where(np.arange(w.Lmax) % 2 == 0, 1.0, 0.0)
    assert (w.with_forms([(8, 0, 1e-12, 1.0)], masks=each).form_layers["act_rep"][0] == 5.0 - each).all()
    assert w.with_forms([(8, 0, 1e-12, 1.0)]).masks is None
    for bad in (-1.0, 6.0, float("nan")):
        with pytest.raises(ValueError, match="masks"):
            w.with_forms([(8, 0, 1e-12, 1.0)], masks=bad)


@gpu
@pytest.mark.parametrize("sp", [0, 1])
def test_masks_keep_their_bytes(sp):
    """A layer with two one-byte masks beside its numbers: in 8 bits it holds the packed numbers and the masks."""
    from paper_2504_03662_b200 import binding as gb
    from paper_2504_03662_b200.search import SearchBuffers
    galv = gb.Galv(0)
    mem = {}
    for masks in (0.0, 2.0):
        w = one_layer(0, sp, 2.0)
        w.layers["act_rep"] += masks
        sb = SearchBuffers(galv, w.with_forms([(8, 0, 0.0, 1.0)], masks=masks))
        sb.eval_costs()
        mem[masks] = sb.mem_q.cpu().numpy()[0, 0] * 64
    kept_masks = 3 * 2 * 2048 * 1024 // (2 if sp else 1)
    assert (mem[2.0] - mem[0.0] == kept_masks).all()                # the same for the plain strategy and the one in 8 bits
    galv.close()
