"""Layer norm and the loss against a teacher in forms that only some sizes take, on the GPU; bounds as in test_gpu_norm_rope_distill.py."""
import pytest

from paper_2010_14501_amd import monet
from test_gpu_norm_rope_distill import EPS, layernorm_call, layernorm_inputs, stream, torch_mod

pytestmark = pytest.mark.gpu

BOTH = pytest.mark.parametrize("dtype", [monet.F32, monet.BF16])


@BOTH
@pytest.mark.parametrize("cols", [16385, 16387, 16391, 16643, 16903, 18433, 24577, 24579, 32769, 32775])
def test_layernorm_of_long_ragged_rows_in_place(dtype, cols):
    """The last, ragged piece of 16 bytes goes back over the end of the piece before it, which in rows of these widths belongs to another wave (in one of the
    two types at least): in place, neither takes a value that the other has stored."""
    torch = torch_mod()
    rows = 700
    (_, tx), (_, tg), (_, tb), (_, tdy) = layernorm_inputs(rows, cols, dtype, monet.F32, 9)
    y, stats, dx, dg, db = layernorm_call(dtype, monet.F32, tx, tg, tb, tdy)
    need = monet.call("monet_layernorm_bwd_workspace_bytes", dtype, rows, cols)
    ws, dg2, db2 = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.empty_like(dg), torch.empty_like(db)
    for _ in range(4):
        got = tx.clone()
        monet.call("monet_layernorm_fwd", stream(), dtype, monet.F32, got.data_ptr(), tg.data_ptr(), tb.data_ptr(), got.data_ptr(), None, rows, cols, cols, cols, EPS)
        assert torch.equal(got, y)
        got = tdy.clone()
        monet.call("monet_layernorm_bwd", stream(), dtype, monet.F32, got.data_ptr(), tx.data_ptr(), tg.data_ptr(), stats.data_ptr(), got.data_ptr(), dg2.data_ptr(),
                   db2.data_ptr(), rows, cols, cols, cols, cols, 0, ws.data_ptr(), need)
        assert torch.equal(got, dx) and torch.equal(dg2, dg) and torch.equal(db2, db)
