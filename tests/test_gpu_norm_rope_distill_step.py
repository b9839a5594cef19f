"""Whole training steps of a transformer graph with layer norm, rotary positions and a loss against a teacher on the GPU, against the oracle's interpreter of
the same schedule."""
import numpy as np
import pytest

from oracle import schedule as osch
from workloads import graphs, schedules, tensors
from paper_2010_14501_amd.runner import StepRunner
from parity_util import ACT_TOL, check_close

pytestmark = pytest.mark.gpu

SCHEDULES = {
    "everything": lambda g: schedules.store_everything_schedule(g),
    "block_outputs": lambda g: schedules.block_output_schedule(g),
    "codes": lambda g: schedules.code_schedule(g),
}
NETS = {
    "ragged": lambda: graphs.transformer(norm=True, rotary=True, teacher=5),
    "long": lambda: graphs.transformer(lens=(150, 0, 3, 71), width=96, heads=6, kv_heads=3, hidden=200, layers=3, vocab=1003, norm=True, rotary=True, teacher=17),
    "labels": lambda: graphs.transformer(lens=(40, 30), norm=True, rotary=True),
    "no_norm": lambda: graphs.transformer(rotary=True, teacher=1),
}


def inputs(g, seed):
    exts, params = tensors.make_inputs(g, seed=seed, gamma_beta="random")
    for ref, name, _, _ in g.exts:
        if name == "teacher_index":
            exts[ref][3], exts[ref][5, 0] = -1, -1
            exts[ref][6, -1] = exts[ref][6, 0]
        elif name == "labels":
            exts[ref][3] = -1
    return exts, params


def compare(g, got, want, tol):
    """Normwise and element-wise, every parameter.  A key bias moves every score of a row alike without rotary positions, and nearly so with slow pairs: its
    gradient is a sum that cancels, rounded to about (length + 16) 2^-24 of its magnitude, and is measured on a tenth of the key weight's."""
    for pid, w in want["grads"].items():
        floor = 0.1 * np.linalg.norm(want["grads"][pid - 1]) if g.params[pid][1].endswith(".k.b") else 0.0
        check_close(got[pid], w, tol, what=g.params[pid][1], floor=floor)


@pytest.mark.parametrize("net", NETS)
@pytest.mark.parametrize("which", SCHEDULES)
def test_step_matches_oracle(net, which):
    g = NETS[net]()
    sch = SCHEDULES[which](g)
    exts, params = inputs(g, 5)
    oe, op = tensors.oracle_inputs(exts, params)
    want = osch.interpret(g.text(), sch.text(), oe, op)
    run = StepRunner(g.text(), sch.text(), exts, params, poison=True)
    assert run.step() == want["peak"]
    assert abs(run.loss_value() - want["loss"]) < ACT_TOL * abs(want["loss"])
    poisoned = run.grads_numpy()
    # fp32 products and sums: 1e-5 and less; codes that round the other way on the GPU move a weight gradient by a step of 2^-7 in few places
    compare(g, poisoned, want, 1e-3 if which == "codes" else 1e-4)
    run.plan.set_poison(False)
    for _ in range(2):
        assert run.step() == want["peak"]
        got = run.grads_numpy()
        assert all(np.array_equal(got[p], poisoned[p]) for p in got)


def test_captured_steps_replay():
    import torch
    g = NETS["long"]()
    exts, params = inputs(g, 6)
    a = StepRunner(g.text(), schedules.code_schedule(g).text(), exts, params)
    b = StepRunner(g.text(), schedules.block_output_schedule(g).text(), exts, params)
    a.step()
    want, loss = a.grads_numpy(), a.loss_value()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step()
    for _ in range(3):
        for t in a.grads:
            t.zero_()
        a.loss.zero_()
        b.step()
        torch.cuda.synchronize()
        graph.replay()
        got = a.grads_numpy()
        assert a.loss_value() == loss and all(np.array_equal(got[p], want[p]) for p in got)


def test_launch_records_name_the_operators():
    g = NETS["ragged"]()
    exts, params = inputs(g, 1)
    run = StepRunner(g.text(), schedules.block_output_schedule(g).text(), exts, params)
    labels = {r[0] for r in run.plan.launches()}
    assert {"layernorm_fwd", "layernorm_bwd", "rope_fwd", "rope_bwd", "lineardistill_fwd", "lineardistill_bwd"} <= labels
