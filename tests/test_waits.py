"""Bounded waits in the kernels that feed the tensor cores, by reading their sources: a wait that runs out cannot be brought about on a GPU without leaving work in flight.

A wait gives up by the waiting lane's own clock.  Where one thread of a warp goes on alone (tc::elect) that is all; where the warp goes on together, into instructions that take all of
its lanes, a lane that gave up by itself would leave the others there for good.  So there the warp decides as one."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2504_03662_b200", "csrc")


def block_end(text, at):
    """Behind the brace that closes the one at `at`."""
    depth = 0
    for i in range(at, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if not depth:
            return i + 1
    raise AssertionError("braces")


def without(text, opening):
    """Without the blocks that `opening` (up to their first brace) begins."""
    while (m := re.search(opening, text)):
        text = text[:m.start()] + text[block_end(text, m.end() - 1):]
    return text


@pytest.mark.parametrize("name", ["galv_expert_matmul.cu", "galv_expert_grad.cu", "galv_mx_matmul.cu", "galv_mx_wgrad.cu"])
def test_warps_decide_as_one_where_they_go_on_together(name):
    with open(os.path.join(CSRC, name)) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    assert text.count("auto waited") >= 1
    text = without(text, r"if \(tc::elect\(\)\) \{")
    text = without(text, r"auto (warp_)?waited = \[&\]\(uint32_t bar, uint32_t parity\) \{")
    together = re.findall(r"[^\n]*\bwaited\([^\n]*", text)
    alone = [line.strip() for line in together if "__shfl_sync(0xffffffffu, (int)(lane == 0 && waited(" not in line]
    assert not alone, alone
    assert "warp_waited(" in text or together
