"""Transformer graphs on the CPU: lowering against the oracle's interpreter, what the 8-bit intermediates save, gradients of the oracle
under every schedule, refusals of graph texts whose shapes the kernels could not take."""
import numpy as np
import pytest

from oracle import network as onet
from oracle import schedule as osch
from test_plan_host import check_against_oracle
from workloads import graphs, schedules, tensors
import paper_2010_14501_amd as M


def test_trace_matches_oracle_on_a_transformer():
    g = graphs.transformer()
    recomputes, peaks = [], []
    for sch in (schedules.store_everything_schedule(g), schedules.store_everything_schedule(g, schedules.CODE_VARIANTS),
                schedules.block_output_schedule(g), schedules.code_schedule(g),
                schedules.block_checkpoint_schedule(g, {1}, schedules.CODE_VARIANTS)):
        plan = check_against_oracle(g, sch)
        recomputes.append(sum(1 for e in plan.trace_tuples() if e[0] == M.RUN_RECOMPUTE))
        peaks.append(plan.exact_peak)
    assert recomputes[0] == recomputes[1] == 0 and min(recomputes[2:]) > 0


def test_codes_hold_less_than_inputs():
    # Bytes a token and layer of width w: everything, 4 (q k v 3w + o w + two sums 2w + ReLU 4w) = 40 w; codes, 4 (o + block output) +
    # 33/32 (q k v o up 5w + down 4w) + mask w / 2 = 17.8 w, and one layer's recomputed tensors at a time.  Eight layers; the vocabulary is
    # small so that its workspace does not count.
    g = graphs.transformer(lens=(1000, 1500, 1596), width=512, heads=8, kv_heads=8, hidden=2048, layers=8, vocab=64)
    full = M.Plan(g.text(), schedules.store_everything_schedule(g).text()).exact_peak
    code = M.Plan(g.text(), schedules.code_schedule(g).text()).exact_peak
    assert code < 0.6 * full, (code, full)


def test_gradients_agree_over_schedules_and_with_differences():
    g = graphs.transformer(lens=(7, 0, 5), width=16, heads=2, kv_heads=1, hidden=24, layers=2, vocab=19)
    exts, params = tensors.make_inputs(g, seed=3)
    exts[-1][2] = -1                                   # a token without a label
    oe, op = tensors.oracle_inputs(exts, params)
    ref = onet.store_everything_step(g.text(), oe, op)
    for sch in (schedules.store_everything_schedule(g), schedules.block_output_schedule(g)):
        got = osch.interpret(g.text(), sch.text(), oe, op)
        assert abs(got["loss"] - ref["loss"]) < 1e-12
        for pid, w in ref["grads"].items():
            assert np.allclose(got["grads"][pid], w, rtol=1e-9, atol=1e-12)
    # inputs in 8 bits: the weight gradients are those of inputs up to 1/128 of their group's maximum away, the rest stays
    code = osch.interpret(g.text(), schedules.code_schedule(g).text(), oe, op)
    assert abs(code["loss"] - ref["loss"]) < 1e-12
    for pid, w in ref["grads"].items():
        d = np.linalg.norm(code["grads"][pid] - w) / np.linalg.norm(w)
        assert d < 0.02, (pid, d)
        if g.params[pid][1].endswith(".b"):
            assert d < 1e-9
    rng = np.random.default_rng(4)
    for pid in range(len(g.params)):
        step = rng.standard_normal(op[pid].shape)
        loss = []
        for h in (1e-5, -1e-5):
            moved = dict(op)
            moved[pid] = op[pid] + h * step
            loss.append(onet.store_everything_step(g.text(), oe, moved)["loss"])
        slope = (loss[0] - loss[1]) / 2e-5
        assert abs(slope - (ref["grads"][pid] * step).sum()) < 1e-6 * (1 + abs(slope)), pid


@pytest.mark.parametrize("old,new,match", [
    ("heads=4 kv_heads=2 dim=16", "heads=4 kv_heads=3 dim=16", "multiple of kv_heads"),
    ("heads=4 kv_heads=2 dim=16", "heads=4 kv_heads=2 dim=8", "tokens x"),
    ("heads=4 kv_heads=2 dim=16", "heads=4 kv_heads=1 dim=16", "keys and values"),
    ("heads=4 kv_heads=2 dim=16", "heads=16 kv_heads=8 dim=4", "multiple of 8"),
    ("seqs=3", "seqs=4", "offsets"),
    ("ext -2 cu_seqlens i32 4", "ext -2 cu_seqlens f32 4", "offsets"),
    ("ext -1 labels i32 64", "ext -1 labels i32 63", "labels"),
    ("lse in=8 par=- shape=4x64", "lse in=8 par=- shape=3x64", "lse"),
    ("act8 in=2 par=- shape=4224", "act8 in=2 par=- shape=4096", "8-bit copy"),
    ("node 8 attention in=2,4,6,-2", "node 8 attention in=2,4,4,-2", "three tensors"),
    ("param 26 head.w 300x64", "param 26 head.w 300x60", "do not fit"),
    ("algo=fused deps=2,4,6,8,9", "algo=fused deps=2,4,6,8", "declared dependencies"),
    ("algo=from_code deps=3", "algo=from_code deps=1", "declared dependencies"),
])
def test_graph_texts_that_do_not_fit_are_refused(old, new, match):
    g = graphs.transformer()
    text = g.text()
    assert old in text, [line for line in text.splitlines() if line.split()[0] in ("ext", "param") or "attention" in line]
    with pytest.raises(M.MonetError, match=match):
        M.Plan(text.replace(old, new, 1), schedules.store_everything_schedule(g).text())
