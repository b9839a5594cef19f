"""The forms of the transformer operators that sizes choose between, special values, and results added to what is there: through the C ABI,
against 64 bits or against the same call without what a test varies.  U and R: half a step of fp32 and bf16, relative to the value."""
import numpy as np
import pytest

from oracle import numerics as nm
from paper_2010_14501_amd import monet
from test_gpu_transformer import R, U, host, linear_ce_bounds, rounded, tdtype, torch_mod, within

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------- the vocabulary loss
def linear_ce_gradients(dtype, tx, tw, labels, start=None, beyond=16 << 20):
    """dx (added to `start` if given) and dw; the workspace is exactly as large as asked for, and what lies behind it is checked."""
    torch = torch_mod()
    (rows, width), vocab = tx.shape, tw.shape[0]
    need = monet.call("monet_linear_ce_workspace_bytes", 1, dtype, rows, width, vocab)
    ws = torch.full((need + beyond,), 255, dtype=torch.uint8, device="cuda")
    loss, lse = torch.empty(1, device="cuda"), torch.empty(rows, device="cuda")
    dx = torch.full_like(tx, float("nan")) if start is None else start.clone()
    dw = torch.full_like(tw, float("nan"))
    s = torch.cuda.current_stream().cuda_stream
    monet.call("monet_linear_ce_fwd", s, dtype, tx.data_ptr(), tw.data_ptr(), labels.data_ptr(), loss.data_ptr(), lse.data_ptr(), rows, width, vocab,
               ws.data_ptr(), need)
    monet.call("monet_linear_ce_bwd", s, dtype, tx.data_ptr(), tw.data_ptr(), labels.data_ptr(), lse.data_ptr(), dx.data_ptr(), dw.data_ptr(), rows,
               width, vocab, 0 if start is None else 1, ws.data_ptr(), need)
    assert (ws[need:] == 255).all()
    return dx, dw


@pytest.mark.parametrize("dtype", [monet.F32, monet.BF16])
@pytest.mark.parametrize("case", [(300, 4096, 100), (257, 64, 700), (130, 72, 257), (2100, 1032, 40), (20, 264, 90), (700, 520, 1500)])
def test_linear_ce_adds_to_dx_and_leaves_dw(case, dtype):
    """Few entries: a single piece and a single range of it, where no sums of ranges are held (the last case has several ranges).  dw is that of the
    call that writes dx, bit for bit, and dx is the sum."""
    torch = torch_mod()
    rows, width, vocab = case
    rng = np.random.default_rng(21)
    x, tx = rounded(rng.standard_normal((rows, width), dtype=np.float32), dtype)
    w, tw = rounded(rng.standard_normal((vocab, width), dtype=np.float32) * np.float32(2.0 / np.sqrt(width)), dtype)
    labels = rng.integers(-1, vocab, rows).astype(np.int32)
    lab = torch.from_numpy(labels).cuda()
    dx, dw = linear_ce_gradients(dtype, tx, tw, lab)
    start = (torch.randn(rows, width, device="cuda") * 0.1).to(tx.dtype)
    added, dw_too = linear_ce_gradients(dtype, tx, tw, lab, start)
    assert torch.equal(dw, dw_too)
    bound = linear_ce_bounds(x, w, labels, dtype)
    want_dx, want_dw = nm.linear_ce_bwd(x, w, labels)
    within(host(dx), want_dx, bound[2], "dx")
    within(host(dw), want_dw, bound[3], "dw")
    total = host(start) + want_dx
    # one more rounding of the sum (fp32: of each piece's sum)
    r = R if dtype == monet.BF16 else 8 * U
    within(host(added), total, bound[2] + 1.1 * r * (np.abs(total) + np.abs(host(start))), "added dx")


# ---------------------------------------------------------------------- 8-bit activations
@pytest.mark.parametrize("dtype", [monet.F32, monet.BF16])
@pytest.mark.parametrize("rows,cols,outs", [(70, 96, 40), (2000, 4090, 2500)])
def test_act8_wgrad_of_groups_up_to_the_largest_numbers(dtype, rows, cols, outs):
    """Groups whose maximum lies at 2^115 to 2^127.98 (the largest that rounds to a code times a power below 2^128 is 63.5 2^122): both forms of
    the weight gradient, directly from the codes and (the larger case in bf16) through the workspace."""
    torch = torch_mod()
    g = torch.Generator(device="cuda")
    g.manual_seed(22)
    groups = -(-cols // 32)
    top = torch.exp2(torch.linspace(115.0, 127.98, groups, device="cuda", dtype=torch.float64))
    x = torch.rand(rows, groups * 32, generator=g, device="cuda", dtype=torch.float64) * 2 - 1
    x[:, ::32] = 1.0
    x = (x.view(rows, groups, 32) * top[:, None]).view(rows, -1)[:, :cols].float().contiguous()
    dy = (torch.randn(rows, outs, generator=g, device="cuda") * (1e-2 / rows)).to(tdtype(dtype))
    code = torch.zeros(monet.call("monet_act8_bytes", rows, cols), dtype=torch.uint8, device="cuda")
    back = torch.empty_like(x)
    monet.call("monet_act8_pack", None, monet.F32, x.data_ptr(), cols, code.data_ptr(), rows, cols)
    monet.call("monet_act8_unpack", None, monet.F32, code.data_ptr(), back.data_ptr(), cols, rows, cols)
    # half a step of a group, 2^e with max / 2^e >= 63.75
    step = torch.exp2(torch.floor(torch.log2(top)) - 5).repeat_interleave(32)[:cols]
    assert torch.isfinite(back).all() and ((back.double() - x.double()).abs() <= 0.5 * step).all()
    need = monet.call("monet_act8_wgrad_workspace_bytes", dtype, rows, cols, outs)
    ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
    dw = torch.full((outs, cols), float("nan"), device="cuda")
    monet.call("monet_act8_wgrad", None, dtype, code.data_ptr(), dy.data_ptr(), dw.data_ptr(), rows, cols, outs, ws.data_ptr(), need)
    want, mag = dy.double().t() @ back.double(), dy.double().abs().t() @ back.double().abs()
    assert torch.isfinite(dw).all()
    assert ((dw.double() - want).abs() <= 1.1 * (3 * rows + 8) * U * mag).all()
