"""Transformer graphs with layer norm, rotary positions and a loss against a teacher, on the CPU: lowering against the oracle's interpreter, gradients of the
oracle under every schedule and by differences, what runs in place, refusals of graph texts that a step could not run."""
import numpy as np
import pytest

from oracle import network as onet
from oracle import schedule as osch
from test_plan_host import check_against_oracle
from workloads import graphs, schedules, tensors
import paper_2010_14501_amd as M

ALL = dict(norm=True, rotary=True, teacher=5)


@pytest.mark.parametrize("parts", [dict(norm=True), dict(rotary=True), dict(teacher=3), ALL])
def test_trace_matches_oracle(parts):
    g = graphs.transformer(**parts)
    for sch in (schedules.store_everything_schedule(g), schedules.store_everything_schedule(g, schedules.CODE_VARIANTS), schedules.block_output_schedule(g),
                schedules.code_schedule(g), schedules.block_checkpoint_schedule(g, {1}, schedules.CODE_VARIANTS)):
        check_against_oracle(g, sch)


def test_rope_runs_in_place_where_its_input_is_not_held():
    g = graphs.transformer(code=False, rotary=True)
    plan = M.Plan(g.text(), schedules.block_output_schedule(g).text())
    ropes = {n.id for n in g.nodes if n.op == "rope"}
    runs = [e for e in plan.trace_tuples() if e[0] in (M.RUN_FWD, M.RUN_RECOMPUTE) and e[2] in ropes]
    assert runs and all(e[4] & 1 for e in runs)


def test_gradients_agree_over_schedules_and_with_differences():
    g = graphs.transformer(lens=(7, 0, 5), width=16, heads=2, kv_heads=1, hidden=24, layers=2, vocab=19, **ALL)
    exts, params = tensors.make_inputs(g, seed=3, gamma_beta="random")
    index = next(r for r, name, _, _ in g.exts if name == "teacher_index")
    exts[index][2] = -1                                # a token without an entry
    exts[index][3, 1] = exts[index][3, 0]
    oe, op = tensors.oracle_inputs(exts, params)
    ref = onet.store_everything_step(g.text(), oe, op)
    for sch in (schedules.store_everything_schedule(g), schedules.block_output_schedule(g)):
        got = osch.interpret(g.text(), sch.text(), oe, op)
        assert abs(got["loss"] - ref["loss"]) < 1e-12
        for pid, w in ref["grads"].items():
            assert np.allclose(got["grads"][pid], w, rtol=1e-9, atol=1e-12)
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


def line(g, start):
    return next(t for t in g.text().splitlines() if t.startswith(start))


@pytest.mark.parametrize("which,old,new,match", [
    ("node 2 layernorm", "eps=1e-05", "eps=0", "eps"),
    ("node 2 layernorm", "eps=1e-05", "eps=nan", "eps"),
    ("node 2 layernorm", "in=1", "in=0", "a node computes"),
    ("node 2 layernorm", "par=2,3", "par=2", "a weight and a bias"),
    ("node 2 layernorm", "par=2,3", "par=2,0", "for each column"),
    ("node 2 layernorm", "64x64", "64x32", "same rows"),
    ("node 3 normstats", "64x2", "64x1", "rows x 2"),
    ("node 3 normstats", "normstats", "lse", "rows x 2"),
    ("node 7 rope", "heads=4 dim=16", "heads=4 dim=8", "tokens x"),
    ("node 7 rope", "heads=4 dim=16", "heads=-4 dim=-16", "bad shape"),
    ("node 7 rope", "rot=16", "rot=15", "rot_dim"),
    ("node 7 rope", "rot=16", "rot=18", "rot_dim"),
    ("node 7 rope", "rot=16", "rot=-2", "rot_dim"),
    ("node 7 rope", "base=10000.0", "base=-1", "base"),
    ("node 7 rope", "factor=1.0", "factor=0", "factor"),
    ("node 7 rope", "high=0.0", "high=4", "blend"),
    ("node 7 rope", "scale=1.0", "scale=inf", "scale"),
    ("node 7 rope", "in=4,-3", "in=4,-1", None),       # any external tensor of that type and size will do
    ("node 7 rope", "in=4,-3", "in=4,-2", "positions"),
    ("node 7 rope", "in=4,-3", "in=4,0", "positions"),
    ("bop 2 layernorm_bwd", "node=2", "node=1", "does not belong"),
    ("bimpl 2 0", "deps=1,3", "deps=1", "declared dependencies"),
    ("bimpl 2 0", "algo=from_input", "algo=from_output", "unknown implementation"),
    ("bop 6 rope_bwd", "rope_bwd", "layernorm_bwd", "does not belong"),
    ("fimpl 2 0", "algo=direct", "inplace=1 algo=direct", "in place"),
])
def test_graph_texts_that_a_step_would_refuse_are_refused_when_loaded(which, old, new, match):
    g = graphs.transformer(code=False, **ALL)
    if which.startswith(("bop", "bimpl")):             # the number that the operator has in this graph
        kind = "rope_bwd" if "rope" in which else "layernorm_bwd"
        k = next(b["k"] for b in g.bops if b["kind"] == kind)
        which = f"{which.split()[0]} {k} {which.split()[2]}"
    if which.startswith("node 7"):
        which = line(g, f"node {next(n.id for n in g.nodes if n.op == 'rope')} rope")
        old = old.replace("in=4,", f"in={which.split('in=')[1].split(',')[0]},")
        new = new.replace("in=4,", f"in={which.split('in=')[1].split(',')[0]},")
    text, sch, at = g.text(), schedules.store_everything_schedule(g).text(), line(g, which)
    assert old in at, at
    changed = text.replace(at, at.replace(old, new, 1), 1)
    if match is None:
        M.Plan(changed, sch)
        return
    with pytest.raises(M.MonetError, match=match):
        M.Plan(changed, sch)


@pytest.mark.parametrize("old,new,match", [
    ("temperature=2.0", "temperature=0", "temperature"), ("temperature=2.0", "temperature=nan", "temperature"), ("top=5", "top=4", "indices"),
    ("top=5", "top=0", "indices"), ("persist=1", "persist=0", "persistent"),
])
def test_a_teachers_loss_that_does_not_fit_is_refused(old, new, match):
    g = graphs.transformer(**ALL)
    at = line(g, f"node {len(g.nodes)} lineardistill")
    assert old in at
    with pytest.raises(M.MonetError, match=match):
        M.Plan(g.text().replace(at, at.replace(old, new), 1), schedules.store_everything_schedule(g).text())
    ext = next(t for t in g.text().splitlines() if "teacher_logits" in t)
    with pytest.raises(M.MonetError, match="logits"):
        M.Plan(g.text().replace(ext, ext.replace("f32", "i32"), 1), schedules.store_everything_schedule(g).text())


@pytest.mark.parametrize("kind", ["layernorm_bwd", "lineardistill_bwd", "lineardistill"])
def test_declared_workspaces_are_checked(kind):
    g = graphs.transformer(**ALL)
    if kind.endswith("bwd"):
        at = line(g, f"bimpl {next(b['k'] for b in g.bops if b['kind'] == kind)} 0")
    else:
        at = line(g, f"fimpl {len(g.nodes)} 0")
    ws = int(at.split(" ws=")[1].split()[0])
    sch = schedules.store_everything_schedule(g).text()
    assert ws > 256
    for less in (0, -5, (ws + 255) // 256 * 256 - 256):
        with pytest.raises(M.MonetError, match="are needed"):
            M.Plan(g.text().replace(at, at.replace(f" ws={ws}", f" ws={less}"), 1), sch)


def test_integer_program_schedules_the_operators():
    """A budget below what storing everything takes: the program recomputes some of them, within the budget by the oracle's model and the executor's."""
    from test_ilp_host import check
    from workloads import ilp
    g = graphs.transformer(lens=(40, 60), layers=1, vocab=40, code=False, **ALL)
    store = M.Plan(g.text(), schedules.store_everything_schedule(g).text()).predicted_peak
    costs = []
    for frac in (1.0, 0.8):
        sch, obj, status = ilp.solve(g, int(frac * store), time_limit=60)
        assert sch is not None, (frac, status)
        check(g, sch, int(frac * store), obj)
        costs.append(obj)
    assert costs[0] < costs[1]
