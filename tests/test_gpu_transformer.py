"""Attention, the vocabulary loss and 8-bit activations on the GPU, through the C ABI, against the oracle in 64 bits.

Bounds are element by element and follow from the arithmetic: U = 2^-24 a rounding in fp32, R = 2^-8 a rounding to bf16 (half a step
relative to the value).  A sum of n products in fp32 is off by at most (n + 2) U times the sum of their magnitudes.  The hardware's
exponential and logarithm are taken as 4 U of their value (documented: one unit in the last place), and a probability
exp(s - lse) carries the absolute error of s and lse."""
import numpy as np
import pytest

from oracle import numerics as nm
from paper_2010_14501_amd import monet

pytestmark = pytest.mark.gpu

U, R = 2.0 ** -24, 2.0 ** -8


def torch_mod():
    import torch
    return torch


def tdtype(dtype):
    torch = torch_mod()
    return torch.bfloat16 if dtype == monet.BF16 else torch.float32


def rounded(a, dtype):
    """The array as the kernels get it, in 64 bits and on the GPU."""
    t = torch_mod().from_numpy(np.ascontiguousarray(a)).to(tdtype(dtype))
    return t.double().numpy(), t.cuda()


def host(t):
    return t.double().cpu().numpy()


def within(got, want, bound, what):
    assert np.isfinite(got).all(), what
    over = np.abs(got - want) - bound
    assert (over <= 0).all(), (what, float(np.abs(got - want).max()), float(over.max()), np.unravel_index(over.argmax(), over.shape))


# ---------------------------------------------------------------------- attention
def attention_bounds(q, k, v, do, cu, scale, dtype):
    """(o, lse, dq, dk, dv) bounds: first-order propagation of the roundings named above, times 1.1 for the higher orders."""
    heads, group, dim = q.shape[1], q.shape[1] // k.shape[1], q.shape[2]
    out = [np.zeros(q.shape), np.zeros((heads, q.shape[0])), np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)]
    rp = R if dtype == monet.BF16 else 0.0
    tiny = 1e-30
    for a, b in zip(cu[:-1], cu[1:]):
        n = b - a
        for h in range(heads if n > 0 else 0):
            kv = h // group
            qs, ks, vs, gs = q[a:b, h], k[a:b, kv], v[a:b, kv], do[a:b, h]
            p, lse = nm._attention_rows(q, k, a, b, h, scale)
            # a score: its sum, the multiplication by scale * log2(e) and the difference from the maximum or lse
            smax = (scale * (np.abs(qs) @ np.abs(ks).T) * np.tri(n)).max(axis=1)
            es = (dim + 8) * U * smax + 4 * U * np.abs(lse)
            # lse: the scores' error, the sum of n terms, the logarithm
            el = es + (n + 16) * U + 4 * U * np.abs(lse)
            ep = (es + el + 8 * U)[:, None] * p                           # of a probability
            o = p @ vs
            eo = (ep + rp * p + (n + 8) * U * p) @ np.abs(vs) + (2 * es + (n + 16) * U)[:, None] * np.abs(o)
            eo = eo + rp * np.abs(o)
            dp = gs @ vs.T
            delta = (p * dp).sum(axis=1)
            edp = (dim + 2) * U * (np.abs(gs) @ np.abs(vs).T)
            edelta = (np.abs(gs) * eo).sum(axis=1) + (dim + 2) * U * (np.abs(gs) * np.abs(o)).sum(axis=1)
            ds = p * (dp - delta[:, None])
            eds = ep * np.abs(dp - delta[:, None]) + p * (edp + edelta[:, None] + 2 * U * (np.abs(dp) + np.abs(delta)[:, None])) + rp * np.abs(ds)
            out[0][a:b, h] = eo
            out[1][h, a:b] = el
            out[2][a:b, h] = scale * ((eds + (n + 4) * U * np.abs(ds)) @ np.abs(ks))
            out[3][a:b, kv] += scale * ((eds + (group * n + 4) * U * np.abs(ds)).T @ np.abs(qs))
            out[4][a:b, kv] += (ep + (rp + (group * n + 4) * U) * p).T @ np.abs(gs)
    if rp:
        for i, w in zip((2, 3, 4), nm.attention_bwd(do, q, k, v, cu, scale)):
            out[i] = out[i] + rp * np.abs(w)
    return [1.1 * b + tiny for b in out]


def attention_call(dtype, q, k, v, do, cu, heads, kv_heads, dim, scale, accumulate=0, start=None, stream=None):
    """Runs both passes on [tokens, ld] tensors (heads in the first columns); outputs begin as `start` (default: -7)."""
    torch = torch_mod()
    n = q.shape[0]
    full = lambda t: torch.full_like(t, -7.0) if start is None else start.clone()[:, :t.shape[1]].contiguous()   # noqa: E731
    o, dq, dk, dv = torch.full_like(do, -7.0), full(q), full(k), full(v)
    lse = torch.full((heads, n), -7.0, device="cuda")
    shape = (len(cu) - 1, n, heads, kv_heads, dim, q.shape[1], k.shape[1], v.shape[1], o.shape[1], scale)
    need = monet.call("monet_attention_bwd_workspace_bytes", dtype, len(cu) - 1, n, heads, kv_heads, dim)
    ws = torch.full((need // 4,), float("nan"), device="cuda")
    s = torch.cuda.current_stream().cuda_stream if stream is None else stream
    monet.call("monet_attention_fwd", s, dtype, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), cu.data_ptr(), *shape)
    monet.call("monet_attention_bwd", s, dtype, do.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(),
               dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), cu.data_ptr(), *shape, accumulate, ws.data_ptr(), need)
    return o, lse, dq, dk, dv


def attention_inputs(rng, n, heads, kv_heads, dim, dtype, pad=0):
    """q, k, v, do in 64 bits and as GPU tensors whose rows are `pad` elements longer than the heads need."""
    ref, gpu = [], []
    for h in (heads, kv_heads, kv_heads, heads):
        a, t = rounded(rng.standard_normal((n, h * dim + pad), dtype=np.float32), dtype)
        ref.append(a[:, :h * dim].reshape(n, h, dim))
        gpu.append(t)
    return ref, gpu


ATTENTION_CASES = [
    # lengths, heads, kv_heads, dim, pad
    ([1], 1, 1, 8, 0),                                    # one token
    ([5, 0, 1, 0, 3], 2, 1, 16, 8),                       # empty sequences between short ones
    ([127, 128, 129], 4, 2, 64, 0),                       # around a workgroup's rows
    ([63, 64, 65, 31, 32, 33], 2, 2, 40, 16),             # around a tile's keys, a dim that fills no strip
    ([300, 17], 8, 2, 128, 8),                            # several tiles, four heads to a key head
    ([257], 3, 3, 96, 24),
    ([1] * 70 + [40] + [2] * 70, 2, 1, 24, 0),            # more sequences than one search step takes
]


@pytest.mark.parametrize("dtype", [monet.F32, monet.BF16])
@pytest.mark.parametrize("case", ATTENTION_CASES)
def test_attention_matches_64_bits(case, dtype):
    lens, heads, kv_heads, dim, pad = case
    torch = torch_mod()
    rng = np.random.default_rng(7)
    before, behind = 3, 5                                  # tokens of no sequence: NaN in, untouched out
    n = sum(lens) + before + behind
    cu_h = before + np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    ref, gpu = attention_inputs(rng, n, heads, kv_heads, dim, dtype, pad)
    for t in gpu:
        t[:before] = float("nan")
        t[n - behind:] = float("nan")
    cu = torch.tensor(cu_h, dtype=torch.int32, device="cuda")
    scale = dim ** -0.5
    got = attention_call(dtype, *gpu, cu, heads, kv_heads, dim, scale)
    q, k, v, do = ref
    o, lse = nm.attention_fwd(q, k, v, cu_h, scale)
    want = [o, lse, *nm.attention_bwd(do, q, k, v, cu_h, scale)]
    bound = attention_bounds(q, k, v, do, cu_h, scale, dtype)
    rows = slice(before, n - behind)
    for name, g, w, b in zip(("o", "lse", "dq", "dk", "dv"), got, want, bound):
        g = host(g)
        if name == "lse":
            assert (g[:, :before] == -7).all() and (g[:, n - behind:] == -7).all()
            within(g[:, rows], w[:, rows], b[:, rows], name)
            continue
        used = w.shape[1] * dim
        assert (g[:before] == -7).all() and (g[n - behind:] == -7).all() and (g[:, used:] == -7).all(), name
        within(g[rows, :used].reshape(w[rows].shape), w[rows], b[rows], name)


@pytest.mark.parametrize("dtype", [monet.F32, monet.BF16])
def test_attention_of_large_scores(dtype):
    """Rows whose running maximum rises in every tile, and rows whose first key holds all the weight."""
    torch = torch_mod()
    rng = np.random.default_rng(8)
    n, heads, kv_heads, dim = 200, 2, 1, 64
    ref, gpu = attention_inputs(rng, n, heads, kv_heads, dim, dtype)
    ramp = np.linspace(0.25, 3.0, n)
    ramp[0] = 4.0
    for i in (0, 1):
        a, gpu[i] = rounded((np.abs(ref[i]) * (ramp[:, None, None] if i else 1.0)).reshape(n, -1).astype(np.float32), dtype)
        ref[i] = a.reshape(n, -1, dim)
    cu = [0, n]
    got = attention_call(dtype, *gpu, torch.tensor(cu, dtype=torch.int32, device="cuda"), heads, kv_heads, dim, 0.5)
    q, k, v, do = ref
    o, lse = nm.attention_fwd(q, k, v, cu, 0.5)
    assert lse.max() > 60
    for name, g, w, b in zip(("o", "lse", "dq", "dk", "dv"), got, [o, lse, *nm.attention_bwd(do, q, k, v, cu, 0.5)],
                             attention_bounds(q, k, v, do, cu, 0.5, dtype)):
        within(host(g).reshape(w.shape), w, b, name)


@pytest.mark.parametrize("dtype", [monet.F32, monet.BF16])
def test_attention_special_values_stay_in_their_sequence(dtype):
    torch = torch_mod()
    rng = np.random.default_rng(9)
    lens, heads, kv_heads, dim = [70, 50, 90], 2, 1, 64
    n = sum(lens)
    ref, gpu = attention_inputs(rng, n, heads, kv_heads, dim, dtype)
    cu = torch.tensor([0, 70, 120, 210], dtype=torch.int32, device="cuda")
    clean = attention_call(dtype, *gpu, cu, heads, kv_heads, dim, 0.125)
    for t, v in zip(gpu, (float("inf"), float("nan"), float("-inf"), float("nan"))):
        t[85, 3] = v
    got = attention_call(dtype, *gpu, cu, heads, kv_heads, dim, 0.125)
    for c, g, name in zip(clean, got, ("o", "lse", "dq", "dk", "dv")):
        if name == "lse":
            c, g = c.t(), g.t()
        assert torch.equal(c[:70], g[:70]) and torch.equal(c[120:], g[120:]), name
        assert not torch.isfinite(g[70:120]).all()


@pytest.mark.parametrize("lens,dim", [([3, 1, 2, 8, 7, 1, 5, 4] * 8, 64), ([127, 129, 64, 65], 128)])
def test_attention_gradients_of_short_sequences(lens, dim):
    """bf16: ds and the result are each rounded once.  A rounding is off by half a step at most and evenly spread: 2^-8 / sqrt(3) of a value at its
    worst in the root of the mean square, sqrt(2) times that for two.  What the rounding of o would add to it has no room."""
    rng = np.random.default_rng(15)
    heads, kv_heads, n = 8, 2, sum(lens)
    ref, gpu = attention_inputs(rng, n, heads, kv_heads, dim, monet.BF16)
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    torch = torch_mod()
    got = attention_call(monet.BF16, *gpu, torch.from_numpy(cu).cuda(), heads, kv_heads, dim, dim ** -0.5)
    q, k, v, do = ref
    want = nm.attention_bwd(do, q, k, v, cu, dim ** -0.5)
    for name, g, w in zip(("dq", "dk", "dv"), got[2:], want):
        w = w.reshape(n, -1)
        assert np.linalg.norm(host(g) - w) < 2.0 ** -8 * (2 / 3) ** 0.5 * np.linalg.norm(w), name


@pytest.mark.parametrize("dtype", [monet.F32, monet.BF16])
def test_attention_repeats_accumulates_and_replays(dtype):
    torch = torch_mod()
    rng = np.random.default_rng(10)
    heads, kv_heads, dim, lens = 4, 2, 64, [150, 0, 77]
    n = sum(lens)
    ref, gpu = attention_inputs(rng, n, heads, kv_heads, dim, dtype)
    cu = torch.tensor([0, 150, 150, 227], dtype=torch.int32, device="cuda")
    one = attention_call(dtype, *gpu, cu, heads, kv_heads, dim, 0.125)
    two = attention_call(dtype, *gpu, cu, heads, kv_heads, dim, 0.125)
    assert all(torch.equal(a, b) for a, b in zip(one, two))
    start = torch.randn(n, heads * dim, device="cuda").to(tdtype(dtype))
    acc = attention_call(dtype, *gpu, cu, heads, kv_heads, dim, 0.125, accumulate=5, start=start)
    r = R if dtype == monet.BF16 else U
    for i, bit in ((2, 1), (3, 0), (4, 1)):
        if not bit:
            assert torch.equal(acc[i], one[i])
            continue
        base = host(start[:, :one[i].shape[1]])
        # one[i] itself is a rounded gradient
        within(host(acc[i]), base + host(one[i]), r * (np.abs(base + host(one[i])) + np.abs(host(one[i]))) * 1.01 + 1e-30, i)
    # captured on another stream, replayed between eager work
    side = torch.cuda.Stream()
    shape = (3, n, heads, kv_heads, dim, heads * dim, kv_heads * dim, kv_heads * dim, heads * dim, 0.125)
    need = monet.call("monet_attention_bwd_workspace_bytes", dtype, 3, n, heads, kv_heads, dim)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    outs = [torch.zeros_like(t) for t in one]
    q, k, v, do = gpu
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        s = torch.cuda.current_stream().cuda_stream
        monet.call("monet_attention_fwd", s, dtype, q.data_ptr(), k.data_ptr(), v.data_ptr(), outs[0].data_ptr(), outs[1].data_ptr(), cu.data_ptr(), *shape)
        monet.call("monet_attention_bwd", s, dtype, do.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), outs[0].data_ptr(), outs[1].data_ptr(),
                   outs[2].data_ptr(), outs[3].data_ptr(), outs[4].data_ptr(), cu.data_ptr(), *shape, 0, ws.data_ptr(), need)
    for _ in range(3):
        for t in outs:
            t.fill_(3.0)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(one, outs))


def test_attention_holds_offsets_to_the_tensors():
    """Offsets beyond the tokens, and descending ones, neither fault nor write outside; the ascending sequences' rows are right."""
    torch = torch_mod()
    rng = np.random.default_rng(11)
    n, heads, dim = 64, 1, 64
    ref, gpu = attention_inputs(rng, n, heads, heads, dim, monet.F32)
    cu = torch.tensor([0, 40, 1 << 30], dtype=torch.int32, device="cuda")
    got = attention_call(monet.F32, *gpu, cu, heads, heads, dim, 0.125)
    want = attention_call(monet.F32, *gpu, torch.tensor([0, 40, 64], dtype=torch.int32, device="cuda"), heads, heads, dim, 0.125)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    cu = torch.tensor([-5, 30, 20, 64], dtype=torch.int32, device="cuda")
    got = attention_call(monet.F32, *gpu, cu, heads, heads, dim, 0.125)
    assert torch.isfinite(got[0]).all()


# ---------------------------------------------------------------------- the vocabulary loss
def linear_ce_call(dtype, x, w, labels, grad=True, accumulate=0, start=None):
    torch = torch_mod()
    rows, width = x.shape
    vocab = w.shape[0]
    need = monet.call("monet_linear_ce_workspace_bytes", 1 if grad else 0, dtype, rows, width, vocab)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    loss, lse = torch.full((1,), -7.0, device="cuda"), torch.full((rows,), -7.0, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    monet.call("monet_linear_ce_fwd", s, dtype, x.data_ptr(), w.data_ptr(), labels.data_ptr(), loss.data_ptr(), lse.data_ptr(), rows, width,
               vocab, ws.data_ptr(), need)
    if not grad:
        return loss, lse
    dx = torch.full_like(x, float("nan")) if start is None else start.clone()
    guard = torch.full((vocab + 2, width), -7.0, device="cuda").to(x.dtype)
    dw = guard[1:-1]
    dw.fill_(float("nan"))
    ws.fill_(255)
    monet.call("monet_linear_ce_bwd", s, dtype, x.data_ptr(), w.data_ptr(), labels.data_ptr(), lse.data_ptr(), dx.data_ptr(), dw.data_ptr(),
               rows, width, vocab, accumulate, ws.data_ptr(), need)
    assert (guard[0] == -7).all() and (guard[-1] == -7).all()
    return loss, lse, dx, dw


def linear_ce_bounds(x, w, labels, dtype):
    rp = R if dtype == monet.BF16 else 0.0
    rows, width = x.shape
    vocab = w.shape[0]
    loss, lse = nm.linear_ce_fwd(x, w, labels)
    logits = x @ w.T
    el_ = (width + 2) * U * (np.abs(x) @ np.abs(w).T).max(axis=1)             # a logit
    m = np.abs(logits).max(axis=1)
    # exponents carry the logit's error and 2 U of the difference; the sum runs over vocab terms; then a logarithm
    else_ = el_ + 4 * U * m + (vocab + 16) * U + 4 * U * np.abs(lse)
    has = (labels >= 0) & (labels < vocab)
    count = max(int(has.sum()), 1)
    eloss = ((else_ + el_ + 2 * U * m)[has]).sum() / count + 2 * U * abs(loss)
    p = np.exp(logits - lse[:, None]) * has[:, None]
    dl = p.copy()
    dl[np.flatnonzero(has), labels[has]] -= 1.0
    dl /= count
    edl = p * (el_ + else_ + 4 * U * m + 8 * U)[:, None] / count + (rp + 4 * U) * np.abs(dl)
    edx = (edl + (vocab + 8) * U * np.abs(dl)) @ np.abs(w)
    edw = (edl + (rows + 8) * U * np.abs(dl)).T @ np.abs(x)
    dx, dw = dl @ w, dl.T @ x
    tiny = 1e-30
    return [1.1 * eloss + tiny, 1.1 * else_ + tiny, 1.1 * (edx + rp * np.abs(dx)) + tiny, 1.1 * (edw + rp * np.abs(dw)) + tiny]


LINEAR_CE_CASES = [
    # rows, width, vocab
    (1, 8, 1), (1, 64, 2), (24, 128, 1009), (130, 72, 257), (3, 200, 5003), (300, 64, 700), (257, 264, 4111), (64, 8, 9000),
]


@pytest.mark.parametrize("dtype", [monet.F32, monet.BF16])
@pytest.mark.parametrize("case", LINEAR_CE_CASES)
def test_linear_ce_matches_64_bits(case, dtype):
    torch = torch_mod()
    rows, width, vocab = case
    rng = np.random.default_rng(12)
    x, tx = rounded(rng.standard_normal((rows, width), dtype=np.float32), dtype)
    w, tw = rounded(rng.standard_normal((vocab, width), dtype=np.float32) * np.float32(2.0 / np.sqrt(width)), dtype)
    labels = rng.integers(0, vocab, rows).astype(np.int32)
    labels[rng.random(rows) < 0.2] = -1
    if rows > 2:
        labels[:3] = [vocab, vocab - 1, 0]               # beyond the vocabulary, its last and its first entry
    got = linear_ce_call(dtype, tx, tw, torch.from_numpy(labels).cuda())
    loss, lse = nm.linear_ce_fwd(x, w, labels)
    want = [np.array([loss]), lse, *nm.linear_ce_bwd(x, w, labels)]
    for name, g, v, b in zip(("loss", "lse", "dx", "dw"), got, want, linear_ce_bounds(x, w, labels, dtype)):
        within(host(g), v, b, name)
    again = linear_ce_call(dtype, tx, tw, torch.from_numpy(labels).cuda())
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    start = torch.randn(rows, width, device="cuda").to(tx.dtype)
    acc = linear_ce_call(dtype, tx, tw, torch.from_numpy(labels).cuda(), accumulate=1, start=start)[2]
    total = host(start) + want[2]
    r = R if dtype == monet.BF16 else (vocab // 64 + 4) * U      # fp32: added to piece by piece
    within(host(acc), total, linear_ce_bounds(x, w, labels, dtype)[2] + 1.1 * r * (np.abs(total) + np.abs(host(start))), "accumulated dx")


@pytest.mark.parametrize("dtype", [monet.F32, monet.BF16])
@pytest.mark.parametrize("case", [(1, 144, 8209), (4, 40, 4096), (5, 264, 4113), (16, 1032, 12304), (17, 520, 4097),
                                  (3, 40, 9001), (4, 264, 8192), (7, 328, 8215), (8, 1288, 8200)])
def test_linear_ce_of_few_rows(case, dtype):
    """Few rows take the input's gradient over ranges of the vocabulary; a row's logits in segments of 4096."""
    test_linear_ce_matches_64_bits(case, dtype)


@pytest.mark.parametrize("dtype", [monet.F32, monet.BF16])
def test_linear_ce_without_a_label(dtype):
    torch = torch_mod()
    x, w = torch.randn(20, 64, device="cuda").to(tdtype(dtype)), torch.randn(300, 64, device="cuda").to(tdtype(dtype))
    loss, lse, dx, dw = linear_ce_call(dtype, x, w, torch.full((20,), -100, dtype=torch.int32, device="cuda"))
    assert loss.item() == 0.0 and not dx.any() and not dw.any() and torch.isfinite(lse).all()


@pytest.mark.parametrize("dtype", [monet.F32, monet.BF16])
def test_linear_ce_of_extreme_logits(dtype):
    """Logits in the thousands, all far below zero in one row, an infinity and a NaN in others: rows do not disturb each other."""
    torch = torch_mod()
    x = torch.zeros(8, 64, device="cuda")
    w = torch.zeros(1000, 64, device="cuda")
    w[:, 0] = torch.linspace(-1.0, 1.0, 1000, device="cuda")
    w[:, 1] = 1.0
    x[0, 0], x[1, 0], x[2, 1], x[3, 1], x[4, 0], x[5, 0] = 4096.0, -4096.0, -3000.0, 3000.0, float("inf"), float("nan")
    x, w = x.to(tdtype(dtype)), w.to(tdtype(dtype))
    lab = torch.tensor([999, 0, 5, 5, -1, -1, 3, 3], dtype=torch.int32, device="cuda")
    loss, lse = linear_ce_call(dtype, x, w, lab, grad=False)
    keep = [0, 1, 2, 3, 6, 7]
    want, wlse = nm.linear_ce_fwd(host(x)[keep], host(w), lab.cpu().numpy()[keep])
    assert np.allclose(host(lse)[keep], wlse, rtol=1e-6) and abs(loss.item() - want) < 1e-3
    assert not np.isfinite(host(lse)[[4, 5]]).any()


def test_linear_ce_in_several_pieces():
    """A workspace for less than the vocabulary: 20000 rows of 13000 logits in bf16 go through in three pieces, the last one ragged."""
    torch = torch_mod()
    rows, width, vocab = 20000, 64, 13005
    need = monet.call("monet_linear_ce_workspace_bytes", 1, monet.BF16, rows, width, vocab)
    assert need < rows * vocab * 2
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = torch.randn(rows, width, generator=g, device="cuda").bfloat16()
    w = (torch.randn(vocab, width, generator=g, device="cuda") * 0.2).bfloat16()
    lab = torch.randint(-1, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    loss, lse, dx, dw = linear_ce_call(monet.BF16, x, w, lab)
    # fp32 on the GPU: the bounds for bf16 outputs are 2^-8 of sums that it holds to 1e-6
    logits = x.float() @ w.float().t()
    ls = torch.logsumexp(logits, 1)
    has = lab >= 0
    at = lab.clamp(min=0).long()
    want = (ls - logits.gather(1, at[:, None])[:, 0])[has].double().mean()
    assert abs(loss.item() - want.item()) < 1e-5 * want.item() and torch.allclose(lse, ls, rtol=1e-5)
    dl = torch.exp(logits - ls[:, None])
    dl.scatter_add_(1, at[:, None], torch.full_like(dl[:, :1], -1.0))
    dl *= (has.float() / has.sum())[:, None]
    for got, ref, mag in ((dx, dl @ w.float(), dl.abs() @ w.float().abs()), (dw, dl.t() @ x.float(), dl.abs().t() @ x.float().abs())):
        assert ((got.float() - ref).abs() <= 1.1 * (R * mag + R * ref.abs()) + 1e-12).all()


# ---------------------------------------------------------------------- 8-bit activations
ACT8_CASES = [(1, 1, 0), (3, 31, 0), (5, 32, 0), (7, 33, 7), (37, 200, 0), (4, 100, 28), (2, 4099, 5), (600, 8, 0)]


@pytest.mark.parametrize("dtype", [monet.F32, monet.BF16])
@pytest.mark.parametrize("case", ACT8_CASES)
def test_act8_is_exact(case, dtype):
    torch = torch_mod()
    rows, cols, pad = case
    rng = np.random.default_rng(13)
    a = rng.standard_normal((rows, cols + pad)) * np.exp2(rng.integers(-6, 6, (rows, 1)))
    a[rng.random(a.shape) < 0.05] *= 2.0 ** -125
    a[rng.random(a.shape) < 0.02] = 0.0
    if rows > 4:
        a[1] *= 2.0 ** 115
        a[2] = 0.0
        a[3, 0] = 127.5 * 2.0 ** 7
        a[4, cols - 1] = np.inf
    x, t = rounded(a.astype(np.float32), dtype)
    nbytes = monet.call("monet_act8_bytes", rows, cols)
    code = torch.full((nbytes + 64,), 77, dtype=torch.uint8, device="cuda")
    y = torch.full_like(t, -7.0)
    monet.call("monet_act8_pack", None, dtype, t.data_ptr(), cols + pad, code.data_ptr(), rows, cols)
    monet.call("monet_act8_unpack", None, dtype, code.data_ptr(), y.data_ptr(), cols + pad, rows, cols)
    want_code, want_byte = nm.act8_pack(x[:, :cols])
    got = code.cpu().numpy()
    n = want_code.size
    assert np.array_equal(got[:n].view(np.int8).reshape(want_code.shape), want_code)
    assert np.array_equal(got[n:nbytes].reshape(want_byte.shape), want_byte) and (got[nbytes:] == 77).all()
    assert np.array_equal(host(y)[:, :cols], nm.act8_unpack(want_code, want_byte, cols), equal_nan=True)
    assert (host(y)[:, cols:] == -7).all()


@pytest.mark.parametrize("dtype", [monet.F32, monet.BF16])
def test_act8_takes_unaligned_rows(dtype):
    torch = torch_mod()
    base = torch.randn(50 * 41 + 1, device="cuda").to(tdtype(dtype))
    x = base[1:].view(50, 41)
    code = torch.zeros(monet.call("monet_act8_bytes", 50, 40), dtype=torch.uint8, device="cuda")
    out = torch.full_like(base, -7.0)
    y = out[1:].view(50, 41)
    monet.call("monet_act8_pack", None, dtype, x.data_ptr(), 41, code.data_ptr(), 50, 40)
    monet.call("monet_act8_unpack", None, dtype, code.data_ptr(), y.data_ptr(), 41, 50, 40)
    assert np.array_equal(host(y)[:, :40], nm.act8_unpack(*nm.act8_pack(host(x)[:, :40]), 40)) and (y[:, 40] == -7).all()


@pytest.mark.parametrize("dtype", [monet.F32, monet.BF16])
@pytest.mark.parametrize("case", [(1, 1, 1), (7, 33, 5), (64, 128, 128), (65, 130, 127), (300, 40, 264), (1030, 200, 9), (2000, 96, 64)])
def test_act8_wgrad_matches_64_bits(case, dtype):
    torch = torch_mod()
    rows, cols, outs = case
    rng = np.random.default_rng(14)
    code_h, byte_h = nm.act8_pack(rng.standard_normal((rows, cols)))
    x = nm.act8_unpack(code_h, byte_h, cols)
    code = torch.from_numpy(np.concatenate([code_h.view(np.uint8).ravel(), byte_h.ravel()])).cuda()
    dy, tdy = rounded(rng.standard_normal((rows, outs), dtype=np.float32), dtype)
    need = monet.call("monet_act8_wgrad_workspace_bytes", dtype, rows, cols, outs)
    ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
    guard = torch.full((outs * cols + 8,), -7.0, device="cuda")
    dw = guard[4:-4].view(outs, cols)
    for shift in (0, 1):                                 # the second time dy lies off a 16-byte boundary
        hold = torch.zeros(rows * outs + shift, device="cuda", dtype=tdtype(dtype))
        src = hold[shift:].view(rows, outs)
        src.copy_(tdy)
        dw.fill_(float("nan"))
        monet.call("monet_act8_wgrad", None, dtype, code.data_ptr(), src.data_ptr(), dw.data_ptr(), rows, cols, outs, ws.data_ptr(), need)
        # codes are exact, so are dy's pieces: only the sums round (fp32: three products to a term, four with the pieces' rest)
        bound = 1.1 * (3 * rows + 8) * U * (np.abs(dy).T @ np.abs(x)) + 1e-30
        within(host(dw), dy.T @ x, bound, shift)
        assert (guard[:4] == -7).all() and (guard[-4:] == -7).all()


@pytest.mark.parametrize("dtype,rows,cols,outs", [(monet.BF16, 3000, 1500, 2050), (monet.BF16, 40000, 4090, 128), (monet.F32, 6100, 4100, 4101)])
def test_act8_wgrad_of_large_layers(dtype, rows, cols, outs):
    """Sizes that go through the workspace as bf16: all rows at once, in several turns, fp32 in three planes."""
    torch = torch_mod()
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    x = torch.randn(rows, cols, generator=g, device="cuda")
    dy = torch.randn(rows, outs, generator=g, device="cuda").to(tdtype(dtype))
    code = torch.zeros(monet.call("monet_act8_bytes", rows, cols), dtype=torch.uint8, device="cuda")
    monet.call("monet_act8_pack", None, monet.F32, x.data_ptr(), cols, code.data_ptr(), rows, cols)
    monet.call("monet_act8_unpack", None, monet.F32, code.data_ptr(), x.data_ptr(), cols, rows, cols)
    need = monet.call("monet_act8_wgrad_workspace_bytes", dtype, rows, cols, outs)
    assert need < 1 << 30
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    dw = torch.full((outs, cols), float("nan"), device="cuda")
    monet.call("monet_act8_wgrad", None, dtype, code.data_ptr(), dy.data_ptr(), dw.data_ptr(), rows, cols, outs, ws.data_ptr(), need)
    want, mag = dy.double().t() @ x.double(), dy.double().abs().t() @ x.double().abs()
    # sums of exact products: (3 rows + 8) U at worst, a random walk in practice
    assert ((dw.double() - want).abs() <= 1.1 * (3 * rows + 8) * U * mag).all()
    assert ((dw.double() - want).norm() / want.norm()).item() < 2e-6


def test_act8_wgrad_of_a_larger_layer():
    test_act8_wgrad_of_large_layers(monet.BF16, 8200, 2050, 1300)


def test_act8_wgrad_stays_in_its_workspace():
    """dy that the products read where it lies (bf16, rows of 16 bytes) takes no other turns than dy that is copied."""
    torch = torch_mod()
    rows, cols, outs = 32000, 4096, 160          # rows of codes alone would fit one turn, with dy beside them they take two
    g = torch.Generator(device="cuda")
    g.manual_seed(6)
    x = torch.randn(rows, cols, generator=g, device="cuda")
    dy = torch.randn(rows * outs + 8, generator=g, device="cuda").bfloat16()
    code = torch.zeros(monet.call("monet_act8_bytes", rows, cols), dtype=torch.uint8, device="cuda")
    monet.call("monet_act8_pack", None, monet.F32, x.data_ptr(), cols, code.data_ptr(), rows, cols)
    monet.call("monet_act8_unpack", None, monet.F32, code.data_ptr(), x.data_ptr(), cols, rows, cols)
    need = monet.call("monet_act8_wgrad_workspace_bytes", monet.BF16, rows, cols, outs)
    ws = torch.full((need + (256 << 20),), 7, dtype=torch.uint8, device="cuda")
    for shift in (0, 1):
        src = dy[shift:shift + rows * outs].view(rows, outs)
        dw = torch.full((outs, cols), float("nan"), device="cuda")
        monet.call("monet_act8_wgrad", None, monet.BF16, code.data_ptr(), src.data_ptr(), dw.data_ptr(), rows, cols, outs, ws.data_ptr(), need)
        assert (ws[need:] == 7).all()
        want, mag = src.double().t() @ x.double(), src.double().abs().t() @ x.double().abs()
        assert ((dw.double() - want).abs() <= 1.1 * (3 * rows + 8) * U * mag).all()


def test_act8_wgrad_of_very_wide_rows():
    """Rows of 2^23 columns and more are beyond the reach of the large products' addresses: the other form takes them."""
    torch = torch_mod()
    rows, cols, outs = 16, (1 << 23) + 5, 160
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    x = torch.randn(rows, cols, generator=g, device="cuda").bfloat16()
    dy = torch.randn(rows, outs, generator=g, device="cuda").bfloat16()
    code = torch.zeros(monet.call("monet_act8_bytes", rows, cols), dtype=torch.uint8, device="cuda")
    monet.call("monet_act8_pack", None, monet.BF16, x.data_ptr(), cols, code.data_ptr(), rows, cols)
    monet.call("monet_act8_unpack", None, monet.BF16, code.data_ptr(), x.data_ptr(), cols, rows, cols)
    need = monet.call("monet_act8_wgrad_workspace_bytes", monet.BF16, rows, cols, outs)
    ws = torch.zeros(max(need, 16), dtype=torch.uint8, device="cuda")
    dw = torch.full((outs, cols), float("nan"), device="cuda")
    monet.call("monet_act8_wgrad", None, monet.BF16, code.data_ptr(), dy.data_ptr(), dw.data_ptr(), rows, cols, outs, ws.data_ptr(), need)
    for at in (slice(0, 5000), slice(cols // 2, cols // 2 + 5000), slice(cols - 5000, cols)):
        want, mag = dy.double().t() @ x[:, at].double(), dy.double().abs().t() @ x[:, at].double().abs()
        assert ((dw[:, at].double() - want).abs() <= 1.1 * (rows + 8) * U * mag).all()
    assert torch.isfinite(dw).all()


def test_act8_wgrad_of_a_marked_group():
    """A group that stands for NaN makes its 32 columns NaN and no others."""
    torch = torch_mod()
    rows, cols, outs = 70, 96, 40
    x = torch.randn(rows, cols, device="cuda")
    x[33, 40] = float("inf")
    code = torch.zeros(monet.call("monet_act8_bytes", rows, cols), dtype=torch.uint8, device="cuda")
    monet.call("monet_act8_pack", None, monet.F32, x.data_ptr(), cols, code.data_ptr(), rows, cols)
    dy = torch.randn(rows, outs, device="cuda").bfloat16()
    need = monet.call("monet_act8_wgrad_workspace_bytes", monet.BF16, rows, cols, outs)
    ws = torch.zeros(max(need, 16), dtype=torch.uint8, device="cuda")
    dw = torch.zeros(outs, cols, device="cuda")
    monet.call("monet_act8_wgrad", None, monet.BF16, code.data_ptr(), dy.data_ptr(), dw.data_ptr(), rows, cols, outs, ws.data_ptr(), need)
    bad = torch.isnan(dw)
    assert bad[:, 32:64].all() and not bad[:, :32].any() and not bad[:, 64:].any()


# ---------------------------------------------------------------------- large and busy
def test_attention_beyond_32_bits():
    """Rows of 2^22 elements that hold every tensor side by side: offsets pass 2^32 elements, and the results are those of compact tensors."""
    torch = torch_mod()
    n, heads, kv_heads, dim, ld = 1200, 2, 1, 64, 1 << 22
    g = torch.Generator(device="cuda")
    g.manual_seed(8)
    cu = torch.tensor([0, 700, 1200], dtype=torch.int32, device="cuda")
    q, do = (torch.randn(n, heads * dim, generator=g, device="cuda").bfloat16() for _ in range(2))
    k, v = (torch.randn(n, kv_heads * dim, generator=g, device="cuda").bfloat16() for _ in range(2))
    want = attention_call(monet.BF16, q, k, v, do, cu, heads, kv_heads, dim, 0.125)
    wide = torch.empty(n, ld, dtype=torch.bfloat16, device="cuda")
    at = {name: wide[:, 1024 * i:1024 * i + t.shape[1]] for i, (name, t) in enumerate(
        dict(q=q, k=k, v=v, do=do, o=q, dq=q, dk=k, dv=v).items())}
    for name, t in dict(q=q, k=k, v=v, do=do).items():
        at[name].copy_(t)
    lse = torch.empty(heads, n, device="cuda")
    need = monet.call("monet_attention_bwd_workspace_bytes", monet.BF16, 2, n, heads, kv_heads, dim)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    shape = (2, n, heads, kv_heads, dim, ld, ld, ld, ld, 0.125)
    p = {name: t.data_ptr() for name, t in at.items()}
    monet.call("monet_attention_fwd", None, monet.BF16, p["q"], p["k"], p["v"], p["o"], lse.data_ptr(), cu.data_ptr(), *shape)
    monet.call("monet_attention_bwd", None, monet.BF16, p["do"], p["q"], p["k"], p["v"], p["o"], lse.data_ptr(), p["dq"], p["dk"], p["dv"],
               cu.data_ptr(), *shape, 0, ws.data_ptr(), need)
    for a, b in zip((at["o"], lse, at["dq"], at["dk"], at["dv"]), want):
        assert torch.equal(a.reshape(-1), b.reshape(-1))


@pytest.mark.parametrize("dtype", [monet.F32, monet.BF16])
def test_linear_ce_beyond_32_bits(dtype):
    """x and dx of more than 2^31 elements: the last rows' lse and gradient, and dw's, against 64 bits."""
    torch = torch_mod()
    rows, width, vocab = 530000, 4096, 40
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    x = torch.randn(rows, width, generator=g, device="cuda", dtype=tdtype(dtype))
    w = (torch.randn(vocab, width, generator=g, device="cuda") * 0.02).to(tdtype(dtype))
    lab = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    loss, lse, dx, dw = linear_ce_call(dtype, x, w, lab)
    wd, total, bound = w.double(), torch.zeros(vocab, width, device="cuda", dtype=torch.float64), torch.zeros(vocab, width, device="cuda", dtype=torch.float64)
    mean = 0.0
    rp = R if dtype == monet.BF16 else 0.0
    for at in range(0, rows, 53000):
        xs, ls = x[at:at + 53000].double(), lab[at:at + 53000].long()
        logits = xs @ wd.t()
        want = torch.logsumexp(logits, 1)
        # a logit is off by (width + 2) U of its terms' sum, at most 0.02 * 4096 or so in all; what follows adds a few U
        err = (width + vocab + 16) * U * (xs.abs() @ wd.abs().t()).max(1).values
        assert ((lse[at:at + 53000].double() - want).abs() <= 1.1 * err).all()
        mean += (want - logits.gather(1, ls[:, None])[:, 0]).sum().item()
        dl = torch.exp(logits - want[:, None])
        edl = dl * (2 * err[:, None] + 8 * U)
        dl[torch.arange(dl.shape[0], device="cuda"), ls] -= 1.0
        edl += (rp + 4 * U) * dl.abs()
        d = dl @ wd / rows
        ed = (edl + (vocab + 8) * U * dl.abs()) @ wd.abs() / rows + rp * d.abs()
        assert ((dx[at:at + 53000].double() - d).abs() <= 1.1 * ed + 1e-30).all()
        total += dl.t() @ xs / rows
        bound += (edl + (rows + 8) * U * dl.abs()).t() @ xs.abs() / rows
    assert ((dw.double() - total).abs() <= 1.1 * (bound + rp * total.abs())).all()
    assert abs(loss.item() - mean / rows) < 1e-5 * mean / rows


def test_calls_on_two_streams_at_once():
    """Calls that share their inputs and run at the same time, each with results and a workspace of its own."""
    torch = torch_mod()
    rng = np.random.default_rng(13)
    heads, dim, n = 4, 64, 2000
    ref, gpu = attention_inputs(rng, n, heads, heads, dim, monet.BF16)
    cu = torch.tensor([0, 900, 2000], dtype=torch.int32, device="cuda")
    x = torch.randn(n, 256, device="cuda")
    w = torch.randn(5003, 256, device="cuda") * 0.1
    lab = torch.randint(-1, 5003, (n,), device="cuda", dtype=torch.int32)
    dy = torch.randn(n, 320, device="cuda")

    def all_of_them():
        code = torch.zeros(monet.call("monet_act8_bytes", n, 256), dtype=torch.uint8, device="cuda")
        need = monet.call("monet_act8_wgrad_workspace_bytes", monet.F32, n, 256, 320)
        ws, dw = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"), torch.empty(320, 256, device="cuda")
        s = torch.cuda.current_stream().cuda_stream
        monet.call("monet_act8_pack", s, monet.F32, x.data_ptr(), 256, code.data_ptr(), n, 256)
        monet.call("monet_act8_wgrad", s, monet.F32, code.data_ptr(), dy.data_ptr(), dw.data_ptr(), n, 256, 320, ws.data_ptr(), need)
        out = [code, dw, *linear_ce_call(monet.F32, x, w, lab), *linear_ce_call(monet.BF16, x.bfloat16(), w.bfloat16(), lab)]
        return out + list(attention_call(monet.BF16, *gpu, cu, heads, heads, dim, 0.125)), ws
    want, _ = all_of_them()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = []
        for st in streams:
            with torch.cuda.stream(st):
                got.append(all_of_them())
        torch.cuda.synchronize()
        for out, _ in got:
            assert all(torch.equal(a, b) for a, b in zip(out, want))
