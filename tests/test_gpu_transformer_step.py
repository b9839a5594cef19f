"""Whole training steps of a transformer graph on the GPU against the oracle's interpreter of the same schedule: attention, linear layers
with and without 8-bit inputs, the vocabulary loss."""
import numpy as np
import pytest

from oracle import schedule as osch
from workloads import graphs, schedules, tensors
from paper_2010_14501_amd.runner import StepRunner
from parity_util import ACT_TOL, check_close

pytestmark = pytest.mark.gpu

SCHEDULES = {
    "everything": lambda g: schedules.store_everything_schedule(g),
    "everything_codes": lambda g: schedules.store_everything_schedule(g, schedules.CODE_VARIANTS),
    "block_outputs": lambda g: schedules.block_output_schedule(g),
    "codes": lambda g: schedules.code_schedule(g),
}
NETS = {
    "ragged": lambda: graphs.transformer(),
    "long": lambda: graphs.transformer(lens=(150, 0, 3, 71), width=96, heads=6, kv_heads=3, hidden=200, layers=3, vocab=1003),
}


def compare(g, got, want, tol):
    """Normwise and element-wise, every parameter.  A key bias moves every score of a row alike, so its gradient vanishes identically:
    the sum over tokens of dk, each of them rounded to about (length + 16) 2^-24 of its magnitude, which is less than 1e-5 of the key
    weight's gradient, the same sum with inputs of about 1 over the width; it is measured on a tenth of that one's norm."""
    for pid, w in want["grads"].items():
        floor = 0.1 * np.linalg.norm(want["grads"][pid - 1]) if g.params[pid][1].endswith(".k.b") else 0.0
        check_close(got[pid], w, tol, what=g.params[pid][1], floor=floor)


@pytest.mark.parametrize("net", NETS)
@pytest.mark.parametrize("which", SCHEDULES)
def test_transformer_step_matches_oracle(net, which):
    g = NETS[net]()
    sch = SCHEDULES[which](g)
    exts, params = tensors.make_inputs(g, seed=5)
    exts[-1][3] = -1
    oe, op = tensors.oracle_inputs(exts, params)
    want = osch.interpret(g.text(), sch.text(), oe, op)
    run = StepRunner(g.text(), sch.text(), exts, params, poison=True)
    assert run.step() == want["peak"]
    assert abs(run.loss_value() - want["loss"]) < ACT_TOL * abs(want["loss"])
    poisoned = run.grads_numpy()
    # fp32 products and sums: 1e-5 and less; codes that round the other way on the GPU move a weight gradient by a step of 2^-7 in few places
    compare(g, poisoned, want, 1e-3 if "codes" in which else 1e-4)
    run.plan.set_poison(False)
    for _ in range(2):
        assert run.step() == want["peak"]
        got = run.grads_numpy()
        assert all(np.array_equal(got[p], poisoned[p]) for p in got)


def test_captured_steps_replay():
    """A step with all of the new operators in a HIP graph, replayed between eager steps of another plan."""
    import torch
    g = NETS["ragged"]()
    exts, params = tensors.make_inputs(g, seed=6)
    a = StepRunner(g.text(), schedules.code_schedule(g).text(), exts, params)
    b = StepRunner(g.text(), schedules.block_output_schedule(g).text(), exts, params)
    a.step()
    want = a.grads_numpy()
    loss = a.loss_value()
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


@pytest.mark.parametrize("which", SCHEDULES)
def test_transformer_step_of_a_padded_batch(which):
    """Offsets that leave tokens in front of the first sequence and behind the last one: attention's output and its gradients are zero there, whatever
    the memory held, so that the linear layers around it sum over zeros."""
    g = NETS["long"]()
    sch = SCHEDULES[which](g)
    exts, params = tensors.make_inputs(g, seed=7)
    cu = next(iter(g.ext_values))
    tokens = exts[cu][-1]
    exts[cu] = np.array([5, 140, 140, 170, tokens - 37], dtype=np.int32)
    exts[-1][:5] = -1
    exts[-1][tokens - 30:] = -1                    # seven tokens of no sequence keep their label
    oe, op = tensors.oracle_inputs(exts, params)
    want = osch.interpret(g.text(), sch.text(), oe, op)
    run = StepRunner(g.text(), sch.text(), exts, params, poison=True)
    for poison in (True, False):
        run.plan.set_poison(poison)
        assert run.step() == want["peak"]
        assert abs(run.loss_value() - want["loss"]) < ACT_TOL * abs(want["loss"])
        compare(g, run.grads_numpy(), want, 1e-3 if "codes" in which else 1e-4)
