"""Strategies that keep in 8 bits or multiply in 4: their price, and the search over them with rates measured from the operators."""
import ctypes as C

import numpy as np
import pytest

from paper_2504_03662_b200 import inputs

gpu = pytest.mark.gpu
FORMS = [(8, 0, 2.5e-13, 1.0), (0, 4, 0.0, 2.75), (8, 4, 2.5e-13, 2.75)]


def priced(w, time_s, mem_bytes, i, l, s):
    """(time, memory) of one entry by the formula of the boundary, in Python's doubles; None without a form."""
    f, sd, ly, p = w.forms[s], w.strat[s], w.layers[0 if w.layers.shape[0] == 1 else i, l], w.inst[i]
    if not f["keep_bits"] and not f["mul_bits"]:
        return None
    h, seq, tp = float(ly["h"]), float(ly["seq"]), float(sd["tp"])
    b = float(p["b"]) / float(sd["batch_div"])
    sbh = seq * b * h
    t, m = time_s, mem_bytes
    if f["keep_bits"]:
        if sd["ckpt"]:
            act = 2.0 * sbh / tp if sd["sp"] else 2.0 * sbh
        elif sd["sp"]:
            act = sbh * (float(ly["act_rep"]) + float(ly["act_tp"])) / tp
        else:
            act = sbh * (float(ly["act_rep"]) + float(ly["act_tp"]) / tp)
        m = m - float(p["act_mult"]) * (act - act * 1.03125 / float(p["bytes_per_elem"]))
        t = t + act * float(f["keep_s_per_byte"])
    if f["mul_bits"]:
        fwd = float(ly["c_lin"]) * b * seq * h * h * (1.0 + float(sd["ckpt"])) / tp / float(p["flops_rate"])
        t = t - (fwd - fwd / float(f["mul_speed"]))
    return t, m


def small(w, B=3, L=5):
    w = w.take(slice(0, B))
    w.Lmax, w.layers, w.L = L, np.ascontiguousarray(w.layers[:, :L]), np.minimum(w.L, [L, L - 2, 1][:B]).astype(np.int32)
    return w


def test_workloads_with_forms():
    w = inputs.config1().with_forms(FORMS)
    assert w.S == 96 and len(w.strat) == len(w.forms) == 96
    assert (w.strat[24:48] == w.strat[:24]).all() and (w.forms["keep_bits"][24:48] == 8).all() and (w.forms["mul_bits"][:48] == 0).all()
    assert w.take(slice(0, 2)).forms is w.forms
    with pytest.raises(ValueError):
        inputs.config0().with_forms(FORMS)                         # measured tables
    with pytest.raises(ValueError):
        inputs.config3().with_forms(FORMS * 2)                     # 64 strategies in 7 forms


def test_refusals_without_a_device():
    from paper_2504_03662_b200 import binding as gb
    lib = gb.load_library()
    sh = gb.make_shape(1, 1, 1, 1)
    assert lib.galv_add_form_cost(None, C.byref(sh), None, None, 0, *([None] * 8)) == gb.ERR_INVALID_ARG
    from paper_2504_03662_b200.search import HostSearch
    with pytest.raises(ValueError):
        HostSearch(None, inputs.config1().with_forms(FORMS))


@gpu
@pytest.mark.parametrize("config", [1, 2, 3])
def test_prices(config, orc):
    import torch
    from paper_2504_03662_b200 import binding as gb
    from paper_2504_03662_b200.search import SearchBuffers
    galv = gb.Galv(0)
    w = small(inputs.CONFIGS[config]()).with_forms(FORMS[:2] if config == 3 else FORMS)
    sb = SearchBuffers(galv, w)
    sb.time_q.fill_(77)
    sb.mem_q.fill_(77)
    sb.step()
    res = sb.results()
    tq, mq = sb.time_q.cpu().numpy(), sb.mem_q.cpu().numpy()
    for i in range(w.B):
        Li = int(w.L[i])
        ts, mb, rt, rm, rx = orc.eval_costs(w.layers[0], w.strat, w.inst[i], Li)
        unit, bins = float(w.inst[i]["time_unit_ns"]), float(w.inst[i]["bin_bytes"])
        want_t, want_m = np.array(rt), np.array(rm)
        for l in range(Li):
            for s in range(w.S):
                p = priced(w, float(ts[l, s]), float(mb[l, s]), i, l, s)
                if p is not None:
                    want_t[l, s], want_m[l, s] = int(np.rint(p[0] * 1e9 / unit)), int(np.ceil(p[1] / bins))
        assert (tq[i, :Li] == want_t).all() and (mq[i, :Li] == want_m).all()
        assert (tq[i, Li:] == 77).all() and (mq[i, Li:] == 77).all()
        ref = orc.search(want_t, want_m, rx, w.M)
        assert res["opt_cost"][i] == ref["opt_cost"] and (res["plan"][i, :Li] == ref["plan"]).all() and res["status"][i] == ref["status"]
    galv.close()


@gpu
def test_forms_that_are_none():
    import torch
    from paper_2504_03662_b200 import binding as gb
    from paper_2504_03662_b200.search import SearchBuffers
    galv = gb.Galv(0)
    for bad in ((4, 0, 0.0, 1.0), (0, 8, 0.0, 1.0), (8, 0, -1.0, 1.0), (8, 0, float("nan"), 1.0), (0, 4, 0.0, 0.0), (0, 4, 0.0, float("inf"))):
        w = small(inputs.config1()).with_forms([bad])
        sb = SearchBuffers(galv, w)
        sb.step()
        assert (sb.results()["status"] & gb.STATUS_BAD_INPUT).all()
        tq = sb.time_q[0].cpu().numpy()
        assert (tq[:, 24:] == -1).all() and (tq[:, :24] >= 0).all()
    lib, h = galv.lib, galv.h
    sh = gb.make_shape(1, 1, 1, 1)
    assert lib.galv_add_form_cost(h, C.byref(sh), None, None, 0, *([None] * 8)) == gb.ERR_INVALID_ARG
    galv.close()


@gpu
def test_measured_rates_make_plans():
    """The path a planner takes: rates from the operators on this device, a plan under a tight budget, the plan's forms carried out."""
    import torch
    from paper_2504_03662_b200 import binding as gb, mx
    from paper_2504_03662_b200.search import SearchBuffers, measure_forms
    galv = gb.Galv(0)
    forms = measure_forms(galv, 1024, 2048)
    assert (forms["keep_bits"] == [8, 0, 8]).all() and (forms["mul_bits"] == [0, 4, 4]).all()
    assert (forms["keep_s_per_byte"][[0, 2]] > 0).all() and (forms["mul_speed"] > 0).all() and np.isfinite(forms["mul_speed"]).all()
    # Without checkpointing: with it the smallest layer is the same in whole 64 MiB bins (12 h^2 * 16 / 8 bytes of state are 1.5 of them, an input of
    # 2 * seq * 8 * h bytes 1, in 8 bits 0.52: three bins either way).
    w = inputs.config1().take(slice(7, 8))
    w.strat = w.strat[w.strat["ckpt"] == 0]
    w.S = len(w.strat)
    plain, held = SearchBuffers(galv, w), SearchBuffers(galv, w.with_forms([FORMS[0]]))
    for sb in (plain, held):
        sb.step()
    budgets = [int(plain.mem_q[0].min(1).values.sum()) - 1, w.M]
    need = int(held.mem_q[0].min(1).values.sum())
    assert need <= budgets[0]                                       # keeping in 8 bits fits where nothing else does
    for sb, status in ((plain, gb.STATUS_INFEASIBLE), (held, 0)):
        sb.backtrack(torch.tensor([budgets[0]], dtype=torch.int32, device="cuda"))
        assert sb.results()["status"][0] == status
    plan = held.results()["plan"][0]
    assert (plan >= w.S).any()                                      # ... and the plan says which layers do
    x = torch.randn(128, 256, device="cuda", dtype=torch.bfloat16)
    weight = torch.randn(64, 256, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    for s in plan[:2]:
        form = held.w.forms[s]
        y = mx.linear(x, weight, four=form["mul_bits"] == 4) if form["keep_bits"] == 8 else torch.nn.functional.linear(x, weight)
        y.sum().backward()
    assert torch.isfinite(weight.grad).all()
    galv.close()
