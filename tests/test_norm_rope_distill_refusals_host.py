"""What a layer norm in a graph refuses: its two gradients are written at the same time, each to a parameter of its own."""
import pytest

from workloads import graphs, schedules
import paper_2010_14501_amd as M


def test_a_layer_norms_weight_and_bias_are_two_parameters():
    g = graphs.transformer(norm=True)
    sch = schedules.store_everything_schedule(g).text()
    n = next(n for n in g.nodes if n.op == "layernorm")
    at = next(t for t in g.text().splitlines() if t.startswith(f"node {n.id} layernorm"))
    pair = f"par={n.pars[0]},{n.pars[1]}"
    assert pair in at
    M.Plan(g.text(), sch)
    M.Plan(g.text().replace(at, at.replace(pair, f"par={n.pars[1]},{n.pars[0]}")), sch)
    with pytest.raises(M.MonetError, match="two parameters"):
        M.Plan(g.text().replace(at, at.replace(pair, f"par={n.pars[0]},{n.pars[0]}")), sch)
