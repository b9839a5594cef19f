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


# ---------------------------------------------------------------------- attention: special values
@pytest.mark.parametrize("dtype", [monet.F32, monet.BF16])
@pytest.mark.parametrize("heads,kv_heads,dim,tokens", [(2, 1, 64, 200), (32, 4, 64, 4224), (2, 1, 128, 200), (32, 4, 128, 4224)])
def test_attention_of_scores_that_overflow_to_minus_infinity(dtype, heads, kv_heads, dim, tokens):
    """The first 150 keys' scores are beyond -3.4e38 for every row behind them: weight 0 there, whichever form the sizes choose (4224 rows and 32
    heads: 128 rows to a workgroup).  The rows before see such keys only, and have no result that means anything."""
    torch = torch_mod()
    rng = np.random.default_rng(23)
    blind = 150
    q = np.zeros((tokens, heads, dim), np.float32)
    k = (rng.standard_normal((tokens, kv_heads, dim)) * 2.0 ** -60).astype(np.float32)
    v = rng.standard_normal((tokens, kv_heads, dim)).astype(np.float32)
    q[:, :, 0] = 2.0 ** 64                             # scores of the others: 2^64 2^-60 n / 8, about 2
    k[:blind, :, :] = 0.0
    k[:blind, :, 0] = -2.0 ** 70
    q, tq = rounded(q.reshape(tokens, -1), dtype)
    k, tk = rounded(k.reshape(tokens, -1), dtype)
    v, tv = rounded(v.reshape(tokens, -1), dtype)
    o, lse = torch.full_like(tq, -7.0), torch.full((heads, tokens), -7.0, device="cuda")
    cu = torch.tensor([0, tokens], dtype=torch.int32, device="cuda")
    monet.call("monet_attention_fwd", torch.cuda.current_stream().cuda_stream, dtype, tq.data_ptr(), tk.data_ptr(), tv.data_ptr(), o.data_ptr(),
               lse.data_ptr(), cu.data_ptr(), 1, tokens, heads, kv_heads, dim, heads * dim, kv_heads * dim, kv_heads * dim, heads * dim, 0.125)
    # all heads of a group are alike, and so are a row's scores but for its key
    for h in range(0, heads, heads // kv_heads):
        kv = h * kv_heads // heads
        s = (0.125 * q.reshape(tokens, heads, dim)[0, h, 0] * k.reshape(tokens, kv_heads, dim)[blind:, kv, 0])
        e = np.exp(s - s.max())
        total = np.cumsum(e)
        w = v.reshape(tokens, kv_heads, dim)[blind:, kv]
        want, want_lse = np.cumsum(e[:, None] * w, 0) / total[:, None], s.max() + np.log(total)
        mag = np.cumsum(e[:, None] * np.abs(w), 0) / total[:, None]
        # a score is one product (two roundings, and the exponential's; the difference from the maximum), the sums run over the keys; bf16 rounds
        # the weights and the result
        n = np.arange(1, tokens - blind + 1)[:, None]
        es = 8 * U * np.abs(s).max() * 2 + (n + 24) * U
        r = R if dtype == monet.BF16 else 0.0
        within(host(o).reshape(tokens, heads, dim)[blind:, h], want, 1.1 * ((2 * es + 2 * r) * mag) + 1e-30, "o")
        within(host(lse)[h, blind:], want_lse, (es + 4 * U * np.abs(want_lse)[:, None])[:, 0] + 1e-30, "lse")
