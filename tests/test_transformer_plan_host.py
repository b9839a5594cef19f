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


@pytest.mark.parametrize("old,new,match", [
    ("seqs=3 scale=0.25", "seqs=3 scale=0", "scale"),
    ("seqs=3 scale=0.25", "seqs=3 scale=-0.25", "scale"),
    ("seqs=3 scale=0.25", "seqs=3 scale=nan", "scale"),
    ("seqs=3 scale=0.25", "seqs=3 scale=inf", "scale"),
    ("deps=2,4,6,8,9 ws=2048", "deps=2,4,6,8,9 ws=1792", "2048 are needed"),
    ("deps=2,4,6,8,9 ws=2048", "deps=2,4,6,8,9 ws=-1000", "2048 are needed"),
    ("fimpl 38 0 algo=pieces ws=77824", "fimpl 38 0 algo=pieces ws=77568", "77824 are needed"),
    ("deps=37 ws=339200", "deps=37 ws=338944", "339200 are needed"),
    ("bop 8 attention_bwd node=8", "bop 8 attention_bwd node=6", "does not belong"),
    ("bop 34 linearce_bwd node=38", "bop 34 linearce_bwd node=37", "does not belong"),
    ("bop 1 linear_wgrad node=1", "bop 1 attention_bwd node=1", "does not belong"),
    ("bimpl 14 0 algo=copy", "bimpl 14 0 algo=from_code", "does not belong"),
    ("node 4 linear in=1 par=4,5", "node 4 linear in=- par=4,5", "one input"),
    ("node 4 linear in=1 par=4,5", "node 4 linear in=1 par=4", "one input"),
])
def test_graph_texts_that_a_step_would_refuse_are_refused_when_loaded(old, new, match):
    """A step that finds something to refuse has launched what comes before it: scales, declared workspaces and the nodes of backward operators
    are looked at when the text is."""
    g = graphs.transformer()
    text = g.text()
    if old.startswith("bimpl 14"):
        old = next(line for line in text.splitlines() if line.startswith("bimpl 14 0 ")).split(" deps=")[0]
    assert text.count(old) >= 1, old
    M.Plan(text, schedules.store_everything_schedule(g).text())
    with pytest.raises(M.MonetError, match=match):
        M.Plan(text.replace(old, new, 1), schedules.store_everything_schedule(g).text())


def test_workspaces_of_codes_are_checked_when_a_graph_is_loaded():
    """From 512 rows on the weight gradient from 8 bits is summed in ranges, which need a workspace: twice 64 x 64 fp32 sums here."""
    g = graphs.transformer(lens=(1024,), layers=1)
    text = g.text()
    old = [line for line in text.splitlines() if "algo=from_code" in line][0]
    ws = int(old.split(" ws=")[1].split()[0])
    assert ws >= 2 * 64 * 64 * 4
    sch = schedules.store_everything_schedule(g).text()
    M.Plan(text, sch)
    for less in (0, ws - 256):
        with pytest.raises(M.MonetError, match="are needed"):
            M.Plan(text.replace(old, old.replace(f" ws={ws}", f" ws={less}"), 1), sch)


def test_attention_of_more_heads_and_tokens_than_a_launch_takes_is_refused_when_loaded():
    """(tokens / 64 + seqs + 8) * heads has to stay below 2^24 - 2^11; nothing of that size is allocated here."""
    g = graphs.transformer(code=False)
    sch = schedules.store_everything_schedule(g).text()
    text = g.text()
    tokens = (1 << 28) + 64
    for kind in ("64x64", "64x32", "64x128"):
        text = text.replace(f" shape={kind}", f" shape={tokens}x{kind[3:]}")
    text = text.replace("shape=4x64", f"shape=4x{tokens}")
    text = text.replace("ext -1 labels i32 64", f"ext -1 labels i32 {tokens}").replace("ext 0 embedded f32 64x64", f"ext 0 embedded f32 {tokens}x64")
    with pytest.raises(M.MonetError, match="too many"):
        M.Plan(text, sch)
