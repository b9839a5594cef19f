"""The forms of the transformer operators that sizes choose between, special values, and results added to what is there: through the C ABI,
against 64 bits or against the same call without what a test varies.  U and R: half a step of fp32 and bf16, relative to the value."""
import numpy as np
import pytest

from oracle import numerics as nm
from paper_2010_14501_amd import monet
from test_gpu_transformer import R, U, attention_call, host, linear_ce_bounds, rounded, tdtype, torch_mod, within

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


@pytest.mark.parametrize("rows,width,vocab", [(1, 1, 1), (5, 1, 37), (9, 3, 5003), (17, 5, 211), (70, 7, 8200), (33, 63, 4099), (130, 65, 129), (6, 131, 9001)])
def test_linear_ce_of_odd_widths_off_16_bytes(rows, width, vocab):
    """fp32 takes any width, and tensors that begin on any word."""
    torch = torch_mod()
    rng = np.random.default_rng(26)
    x, tx = rounded(rng.standard_normal((rows, width), dtype=np.float32), monet.F32)
    w, tw = rounded(rng.standard_normal((vocab, width), dtype=np.float32) * np.float32(2.0 / np.sqrt(width)), monet.F32)
    labels = rng.integers(-1, vocab, rows).astype(np.int32)
    lab = torch.from_numpy(labels).cuda()
    want = nm.linear_ce_bwd(x, w, labels)
    bound = linear_ce_bounds(x, w, labels, monet.F32)[2:]
    for off in (0, 1, 3):
        def shifted(t):
            hold = torch.full((t.numel() + 8,), -7.0, device="cuda")
            at = hold[off:off + t.numel()].view(t.shape)
            at.copy_(t)
            return hold, at
        (_, ax), (_, aw), (hx, dx), (hw, dw) = shifted(tx), shifted(tw), shifted(tx), shifted(tw)
        need = monet.call("monet_linear_ce_workspace_bytes", 1, monet.F32, rows, width, vocab)
        ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
        loss, lse = torch.empty(1, device="cuda"), torch.empty(rows, device="cuda")
        s = torch.cuda.current_stream().cuda_stream
        monet.call("monet_linear_ce_fwd", s, monet.F32, ax.data_ptr(), aw.data_ptr(), lab.data_ptr(), loss.data_ptr(), lse.data_ptr(), rows, width,
                   vocab, ws.data_ptr(), need)
        monet.call("monet_linear_ce_bwd", s, monet.F32, ax.data_ptr(), aw.data_ptr(), lab.data_ptr(), lse.data_ptr(), dx.data_ptr(), dw.data_ptr(),
                   rows, width, vocab, 0, ws.data_ptr(), need)
        for name, hold, got, ref, b in (("dx", hx, dx, want[0], bound[0]), ("dw", hw, dw, want[1], bound[1])):
            within(host(got), ref, b, (name, off))
            assert (hold[:off] == -7).all() and (hold[off + got.numel():] == -7).all()


def linear_ce_reference(x, w, lab, dtype, rows_at_a_time):
    """On the GPU, in 64 bits, some rows at a time: (loss, lse, dx, dw) and bounds, from the same arithmetic as linear_ce_bounds."""
    torch = torch_mod()
    rp = R if dtype == monet.BF16 else 0.0
    (rows, width), vocab = x.shape, w.shape[0]
    wd = w.double()
    wa = wd.abs()
    count = max(1, int(((lab >= 0) & (lab < vocab)).sum()))
    zero = lambda *s: torch.zeros(*s, dtype=torch.float64, device="cuda")   # noqa: E731
    out, bound = [zero(1), zero(rows), zero(rows, width), zero(vocab, width)], [zero(1), zero(rows), zero(rows, width), zero(vocab, width)]
    for a in range(0, rows, rows_at_a_time):
        part = slice(a, min(rows, a + rows_at_a_time))
        xs, ls = x[part].double(), lab[part].long()
        logits = xs @ wd.t()
        lse = torch.logsumexp(logits, 1)
        m = logits.abs().amax(1)
        el = (width + 2) * U * (xs.abs() @ wa.t()).amax(1)
        els = el + 4 * U * m + (vocab + 16) * U + 4 * U * lse.abs()
        has = torch.nonzero((ls >= 0) & (ls < vocab))[:, 0]
        out[0] += (lse[has] - logits[has, ls[has]]).sum() / count
        bound[0] += (els + el + 2 * U * m)[has].sum() / count
        out[1][part], bound[1][part] = lse, els
        p = torch.zeros_like(logits)
        p[has] = torch.exp(logits[has] - lse[has, None])
        edl = p * (el + els + 4 * U * m + 8 * U)[:, None]
        p[has, ls[has]] -= 1.0
        edl += (rp + 4 * U) * p.abs()
        out[2][part] = p @ wd / count
        bound[2][part] = (edl + (vocab + 8) * U * p.abs()) @ wa / count
        out[3] += p.t() @ xs / count
        bound[3] += (edl + (rows + 8) * U * p.abs()).t() @ xs.abs() / count
        del logits, p, edl
    bound[0] += 2 * U * out[0].abs()
    for i in (2, 3):
        bound[i] += rp * out[i].abs()
    return out, [1.1 * b + 1e-30 for b in bound]


@pytest.mark.parametrize("dtype,rows,width,vocab,at_a_time,sums", [
    # 13 pieces of 61696 entries in 16 ranges each, the last one of 58485 in 15 (the offsets of its sums are the first one's)
    (monet.BF16, 2048, 8, 798837, 128, 16),
    # two pieces of 50176 entries, each in 8 ranges of large tiles
    (monet.BF16, 2048, 1024, 100001, 512, 8),
    # three pieces of 3328 entries and one of three
    (monet.F32, 20000, 64, 9507, 2500, None),
    # pieces whose weights stay below 4 GiB, and the rest: 5120 and 980 entries (those of a few rows, which are read directly, and those of more)
    (monet.F32, 33, 200000, 6100, 33, None),
    (monet.F32, 7, 200000, 6100, 7, None),
])
def test_linear_ce_over_pieces_and_ranges(dtype, rows, width, vocab, at_a_time, sums):
    """Several pieces of the vocabulary, with dx's sums held over several ranges of each, or in large tiles; dx written and added to."""
    torch = torch_mod()
    g = torch.Generator(device="cuda")
    g.manual_seed(25)
    x = torch.randn(rows, width, generator=g, device="cuda").to(tdtype(dtype))
    w = torch.empty(vocab, width, dtype=tdtype(dtype), device="cuda")
    for a in range(0, vocab, 1 << 15):
        part = w[a:a + (1 << 15)]
        part.copy_(torch.randn(part.shape, generator=g, device="cuda") * (1.5 * width ** -0.5))
    lab = torch.randint(-1, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    lab[0] = vocab - 1
    if sums:      # the workspace holds dx's sums of so many ranges, and a piece of the gradient besides
        need = monet.call("monet_linear_ce_workspace_bytes", 1, dtype, rows, width, vocab)
        assert need < rows * vocab * 2 and need >= sums * rows * width * 4 + rows * 2 * vocab // -(-vocab * rows * 2 // (256 << 20))
    loss, lse = torch.empty(1, device="cuda"), torch.empty(rows, device="cuda")
    dx, dw = linear_ce_gradients(dtype, x, w, lab)
    need = monet.call("monet_linear_ce_workspace_bytes", 0, dtype, rows, width, vocab)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    monet.call("monet_linear_ce_fwd", s, dtype, x.data_ptr(), w.data_ptr(), lab.data_ptr(), loss.data_ptr(), lse.data_ptr(), rows, width, vocab,
               ws.data_ptr(), need)
    del ws
    want, bound = linear_ce_reference(x, w, lab, dtype, at_a_time)
    for name, got, ref, b in zip(("loss", "lse", "dx", "dw"), (loss, lse, dx, dw), want, bound):
        over = (got.double() - ref).abs() - b
        assert (over <= 0).all(), (name, over.max().item())
        del over
    start = (torch.randn(rows, width, generator=g, device="cuda") * 0.1).to(x.dtype)
    added, dw_too = linear_ce_gradients(dtype, x, w, lab, start)
    assert torch.equal(dw, dw_too)
    total = start.double() + want[2]
    r = R if dtype == monet.BF16 else 8 * U      # fp32: a rounding for each piece
    assert ((added.double() - total).abs() <= bound[2] + 1.1 * r * (total.abs() + start.double().abs())).all()


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


# ---------------------------------------------------------------------- attention: the forms that sizes choose between
def attention_group(q, k, v, do, scale, dtype):
    """One sequence and one key / value head with its group of query heads, in 64 bits on the GPU: (results, bounds) of o [group, n, dim], lse
    [group, n], dq, dk [n, dim], dv.  The bounds propagate to first order, times 1.1 for the rest: a sum of n products in fp32 is off by (n + 2) U
    of their magnitudes, exponential and logarithm by 4 U, bf16 rounds the probabilities, ds and the results by R."""
    torch = torch_mod()
    group, n, dim = q.shape
    rp = R if dtype == monet.BF16 else 0.0
    seen = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
    zero = lambda *s: torch.zeros(*s, dtype=torch.float64, device="cuda")   # noqa: E731
    out = [zero(group, n, dim), zero(group, n), zero(group, n, dim), zero(n, dim), zero(n, dim)]
    bound = [t.clone() for t in out]
    for h in range(group):
        qs, gs = q[h], do[h]
        s = (scale * (qs @ k.t())).masked_fill(~seen, float("-inf"))
        lse = torch.logsumexp(s, 1)
        p = torch.exp(s - lse[:, None])
        o, dp = p @ v, gs @ v.t()
        delta = (p * dp).sum(1, keepdim=True)
        ds = p * (dp - delta)
        out[0][h], out[1][h], out[2][h] = o, lse, scale * (ds @ k)
        out[3] += scale * (ds.t() @ qs)
        out[4] += p.t() @ gs
        smax = (scale * (qs.abs() @ k.abs().t()) * seen).amax(1)
        es = (dim + 8) * U * smax + 4 * U * lse.abs()
        el = es + (n + 16) * U + 4 * U * lse.abs()
        ep = (es + el + 8 * U)[:, None] * p
        eo = (ep + (rp + (n + 8) * U) * p) @ v.abs() + (2 * es + (n + 16) * U)[:, None] * o.abs()
        eo = eo + rp * o.abs()
        edp = (dim + 2) * U * (gs.abs() @ v.abs().t())
        edelta = (gs.abs() * eo).sum(1, keepdim=True) + (dim + 2) * U * (gs.abs() * o.abs()).sum(1, keepdim=True)
        eds = ep * (dp - delta).abs() + p * (edp + edelta + 2 * U * (dp.abs() + delta.abs())) + rp * ds.abs()
        bound[0][h], bound[1][h] = eo, el
        bound[2][h] = scale * ((eds + (n + 4) * U * ds.abs()) @ k.abs()) + rp * out[2][h].abs()
        bound[3] += scale * ((eds + (group * n + 4) * U * ds.abs()).t() @ qs.abs())
        bound[4] += (ep + (rp + (group * n + 4) * U) * p).t() @ gs.abs()
    bound[3] += rp * out[3].abs()
    bound[4] += rp * out[4].abs()
    return out, [1.1 * b + 1e-30 for b in bound]


LONG, TAIL = [2125, 1, 0, 1990, 129, 300], [0] * 20
FORMS = {
    # name: lengths, heads, kv_heads, dim, whether dk and dv are summed over ranges (fp32, bf16)
    "128_rows_128_keys_64": (LONG, 32, 32, 64, (False, False)),              # from 1024 workgroups of 128 rows (keys) on
    "128_rows_128_keys_128": (LONG, 32, 32, 128, (False, False)),
    "128_rows_ranges_40": (LONG, 32, 8, 40, (True, True)),
    "128_rows_ranges_128": (LONG, 32, 8, 128, (True, True)),
    "128_rows_ranges_of_padded_offsets": (LONG + TAIL, 32, 8, 96, (True, True)),
    "64_rows_32_keys_ranges_64": ([2100, 40, 0, 65], 2, 1, 64, (True, True)),
    "64_rows_32_keys_ranges_128": ([1500, 700], 4, 1, 128, (True, True)),
    "64_rows_32_keys_padded_offsets": ([0, 0, 1800, 3] + [0] * 60, 6, 2, 64, (True, True)),
    "64_rows_32_keys": ([500, 300, 224, 64, 7], 16, 16, 72, (True, False)),
    "64_rows_128_keys_ranges": ([1300, 1295], 32, 8, 128, (True, True)),     # the mean length gives ranges for two workgroups to a CU
    "short_128_rows": ([100] * 41 + [17, 1, 32, 128, 255], 32, 8, 64, (True, True)),
}


@pytest.mark.parametrize("dtype", [monet.F32, monet.BF16])
@pytest.mark.parametrize("form", FORMS)
def test_attention_forms_match_64_bits(form, dtype):
    """Every form of the three kernels, with tokens in front of the sequences and behind them, rows longer than the heads need, written and added to;
    every row of the first, the last and a middle key head and of their groups."""
    torch = torch_mod()
    lens, heads, kv_heads, dim, ranges = FORMS[form]
    before, behind, pad = 3, 5, 8
    n = sum(lens) + before + behind
    cu_h = [before + sum(lens[:i]) for i in range(len(lens) + 1)]
    cu = torch.tensor(cu_h, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(24)
    gpu = []
    for h in (heads, kv_heads, kv_heads, heads):
        t = torch.randn(n, h * dim + pad, generator=g, device="cuda").to(tdtype(dtype))
        t[:before] = float("nan")
        t[n - behind:] = float("nan")
        gpu.append(t)
    scale = dim ** -0.5
    need = monet.call("monet_attention_bwd_workspace_bytes", dtype, len(lens), n, heads, kv_heads, dim)
    assert (need >= 4 * n * kv_heads * dim * 4) == ranges[dtype], need
    one = attention_call(dtype, *gpu, cu, heads, kv_heads, dim, scale)
    start = torch.randn(n, heads * dim + pad, generator=g, device="cuda").to(tdtype(dtype))
    added = attention_call(dtype, *gpu, cu, heads, kv_heads, dim, scale, accumulate=7, start=start)
    names = ("o", "lse", "dq", "dk", "dv")
    for name, t, u in zip(names, one, added):
        if name == "lse":
            assert (t[:, :before] == -7).all() and (t[:, n - behind:] == -7).all()
            assert torch.equal(t, u)
            continue
        used = (heads if name in ("o", "dq") else kv_heads) * dim
        assert (t[:before] == -7).all() and (t[n - behind:] == -7).all() and (t[:, used:] == -7).all(), name
        if name == "o":
            assert torch.equal(t, u)
            continue
        base = start[:, :t.shape[1]]
        rows = slice(before, n - behind)
        assert torch.equal(u[:before], base[:before]) and torch.equal(u[n - behind:], base[n - behind:]) and torch.equal(u[:, used:], base[:, used:])
        # t is the rounded gradient, u the rounded sum
        x, y, z = base[rows, :used].double(), t[rows, :used].double(), u[rows, :used].double()
        r = R if dtype == monet.BF16 else U
        assert ((z - x - y).abs() <= 1.01 * r * ((x + y).abs() + y.abs()) + 1e-30).all(), name
    group = heads // kv_heads
    split = lambda t, h: t[:, :h * dim].view(n, h, dim).transpose(0, 1).double()   # noqa: E731
    q, do, o, dq = (split(t, heads) for t in (gpu[0], gpu[3], one[0], one[2]))
    k, v, dk, dv = (split(t, kv_heads) for t in (gpu[1], gpu[2], one[3], one[4]))
    for kv in sorted({0, kv_heads // 2, kv_heads - 1}):
        hs = slice(kv * group, (kv + 1) * group)
        for a, b in zip(cu_h[:-1], cu_h[1:]):
            if a == b:
                continue
            want, bound = attention_group(q[hs, a:b], k[kv, a:b], v[kv, a:b], do[hs, a:b], scale, dtype)
            got = (o[hs, a:b], one[1][hs, a:b].double(), dq[hs, a:b], dk[kv, a:b], dv[kv, a:b])
            for name, x, w, e in zip(names, got, want, bound):
                over = (x - w).abs() - e
                assert (over <= 0).all(), (name, kv, a, b, (x - w).abs().max().item(), over.max().item())


# ---------------------------------------------------------------------- captured calls
@pytest.mark.parametrize("dtype", [monet.F32, monet.BF16])
def test_captured_calls_replay(dtype):
    """The vocabulary loss over several pieces, 8-bit activations and (bf16: both forms of) their weight gradient in two graphs that share one workspace,
    replayed in turn between eager calls with another one: every replay gives the eager results, and follows inputs that change."""
    torch = torch_mod()
    g = torch.Generator(device="cuda")
    g.manual_seed(27)
    rows, width, vocab, outs = 3000, 1504, 50001, 5000
    mk = lambda *s: torch.randn(*s, generator=g, device="cuda").to(tdtype(dtype))   # noqa: E731
    x, w, dy = mk(rows, width), mk(vocab, width) * width ** -0.5, mk(rows, outs)
    lab = torch.randint(-1, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    narrow = dy[:, :96].contiguous()
    need = max(monet.call("monet_linear_ce_workspace_bytes", 1, dtype, rows, width, vocab),
               monet.call("monet_act8_wgrad_workspace_bytes", dtype, rows, width, outs), monet.call("monet_act8_wgrad_workspace_bytes", dtype, rows, width, 96))
    code_bytes = monet.call("monet_act8_bytes", rows, width)

    def outputs():
        f = lambda *s: torch.full(s, -7.0, device="cuda")   # noqa: E731
        return dict(loss=f(1), lse=f(rows), dx=torch.full_like(x, -7.0), dw=torch.full_like(w, -7.0)), dict(
            code=torch.full((code_bytes,), 9, dtype=torch.uint8, device="cuda"), y=torch.full_like(x, -7.0), wide=f(outs, width), narrow=f(96, width))

    def loss_calls(t, ws):
        s = torch.cuda.current_stream().cuda_stream
        monet.call("monet_linear_ce_fwd", s, dtype, x.data_ptr(), w.data_ptr(), lab.data_ptr(), t["loss"].data_ptr(), t["lse"].data_ptr(), rows, width,
                   vocab, ws.data_ptr(), need)
        monet.call("monet_linear_ce_bwd", s, dtype, x.data_ptr(), w.data_ptr(), lab.data_ptr(), t["lse"].data_ptr(), t["dx"].data_ptr(),
                   t["dw"].data_ptr(), rows, width, vocab, 0, ws.data_ptr(), need)

    def code_calls(t, ws):
        s = torch.cuda.current_stream().cuda_stream
        monet.call("monet_act8_pack", s, dtype, x.data_ptr(), width, t["code"].data_ptr(), rows, width)
        monet.call("monet_act8_unpack", s, dtype, t["code"].data_ptr(), t["y"].data_ptr(), width, rows, width)
        for name, src, n in (("wide", dy, outs), ("narrow", narrow, 96)):
            monet.call("monet_act8_wgrad", s, dtype, t["code"].data_ptr(), src.data_ptr(), t[name].data_ptr(), rows, width, n, ws.data_ptr(), need)

    shared, other = (torch.full((need,), 255, dtype=torch.uint8, device="cuda") for _ in range(2))
    a, b = outputs()
    graphs = []
    torch.cuda.synchronize()
    for calls, t in ((loss_calls, a), (code_calls, b)):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            calls(t, shared)
        graphs.append(graph)
    for turn in range(3):
        ea, eb = outputs()
        for t in (a, b):
            for v in t.values():
                v.fill_(5)
        for graph, calls, t in zip(graphs, (loss_calls, code_calls), (ea, eb)):
            graph.replay()
            calls(t, other)
        torch.cuda.synchronize()
        for t, e in ((a, ea), (b, eb)):
            for name in t:
                assert torch.equal(t[name], e[name]), (turn, name)
        x.mul_(1.5)
        lab.copy_(lab.flip(0))
