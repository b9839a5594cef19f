"""Layer norm, rotary positions and the loss against a teacher's top logits, without a GPU: pins of the oracle's definitions (hand-worked values,
differences), the frequency tables, and what the entry points refuse before anything is enqueued (the addresses are never read)."""
import numpy as np
import pytest

from oracle import numerics as nm
from paper_2010_14501_amd import monet

P = 1 << 20


def fd(f, x, i, h=1e-5):
    a, b = x.copy(), x.copy()
    a[i] += h
    b[i] -= h
    return (f(a) - f(b)) / (2 * h)


def refused(match, name, *args):
    with pytest.raises(monet.MonetError, match=match):
        monet.call(name, *args)


# ---------------------------------------------------------------------- the oracle
def test_layernorm_by_hand_and_by_differences():
    y, mean, rstd = nm.layernorm_fwd(np.array([[1.0, 3.0], [5.0, 5.0]]), np.array([2.0, 2.0]), np.array([0.0, 1.0]), 3.0)
    assert np.allclose(mean, [2, 5]) and np.allclose(rstd, [0.5, 3 ** -0.5]) and np.allclose(y, [[-1, 2], [0, 1]])
    rng = np.random.default_rng(0)
    x, dy, gamma, beta = rng.standard_normal((3, 5)), rng.standard_normal((3, 5)), rng.standard_normal(5), rng.standard_normal(5)
    f = lambda a, g, b: (dy * nm.layernorm_fwd(a, g, b, 0.1)[0]).sum()   # noqa: E731
    dx, dgamma, dbeta = nm.layernorm_bwd(dy, x, gamma, 0.1)
    for i in np.ndindex(x.shape):
        assert abs(fd(lambda t: f(t, gamma, beta), x, i) - dx[i]) < 1e-8
    for i in range(5):
        assert abs(fd(lambda t: f(x, t, beta), gamma, i) - dgamma[i]) < 1e-8
        assert abs(fd(lambda t: f(x, gamma, t), beta, i) - dbeta[i]) < 1e-8


def test_rope_by_hand_and_by_differences():
    x = np.arange(1.0, 7.0).reshape(1, 1, 6)
    quarter = np.array([np.pi / 2, np.pi])
    assert np.allclose(nm.rope_fwd(x, np.array([1]), quarter, True), [[[-2, 1, -3, -4, 5, 6]]])
    assert np.allclose(nm.rope_fwd(x, np.array([1]), quarter, False, 2.0), [[[-6, -4, 2, -8, 5, 6]]])
    rng = np.random.default_rng(1)
    x, dy, at, f = rng.standard_normal((3, 2, 8)), rng.standard_normal((3, 2, 8)), np.array([0, 7, -3]), nm.rope_freqs(6, 100.0)
    for interleaved in (False, True):
        dx = nm.rope_bwd(dy, at, f, interleaved, 1.3)
        for i in np.ndindex(x.shape):
            assert abs(fd(lambda t: (dy * nm.rope_fwd(t, at, f, interleaved, 1.3)).sum(), x, i) - dx[i]) < 1e-8


@pytest.mark.parametrize("known", [False, True])
def test_linear_distill_by_hand_and_by_differences(known):
    # uniform logits over five entries, the teacher 3 : 1 over two of them
    loss, lse, mass, delta = nm.linear_distill_fwd(np.ones((2, 2)), np.zeros((5, 2)), np.array([[1, 4, 7], [-1, 5, 9]]),
                                                   np.array([[2 * np.log(3.0), 0.0, 9.0], [1.0, 2.0, 3.0]]), 2.0)
    assert np.isclose(loss, 4 * (0.75 * np.log(3.75) + 0.25 * np.log(1.25))) and np.allclose(lse, np.log(5.0))
    assert np.allclose(mass, [1, 0]) and np.allclose(delta, [[0.2 - 0.75, 0.2 - 0.25, 0], [0, 0, 0]])
    rng = np.random.default_rng(2)
    x, w, target = rng.standard_normal((6, 4)), rng.standard_normal((9, 4)), 2 * rng.standard_normal((6, 3))
    index = np.array([[0, 8, 3], [2, 2, 5], [-1, 9, 100], [4, -1, 4], [1, 6, 7], [7, 0, 1]])      # twice the same, none, out of range
    target[4, 1] = -np.inf
    known = 2.0 + rng.random(6) if known else None
    f = lambda a, b: nm.linear_distill_fwd(a, b, index, target, 1.7, known)[0]   # noqa: E731
    dx, dw = nm.linear_distill_bwd(x, w, index, target, 1.7, known)
    for i in np.ndindex(x.shape):
        assert abs(fd(lambda t: f(t, w), x, i) - dx[i]) < 1e-8
    for i in np.ndindex(w.shape):
        assert abs(fd(lambda t: f(x, t), w, i) - dw[i]) < 1e-8
    # one entry a row: the cross entropy of that label
    lab = np.array([0, 8, -1, 3, 4, 3])
    one = nm.linear_distill_fwd(x, w, lab[:, None], target[:, 2:], 1.0)
    assert np.isclose(one[0], nm.linear_ce_fwd(x, w, lab)[0])
    for a, b in zip(nm.linear_distill_bwd(x, w, lab[:, None], target[:, 2:], 1.0), nm.linear_ce_bwd(x, w, lab)):
        assert np.allclose(a, b)


# ---------------------------------------------------------------------- frequencies
@pytest.mark.parametrize("args", [(128, 1e4), (2, 1e4), (64, 5e5, 8.0), (96, 1e4, 4.0, 8192.0, 1.0, 4.0), (512, 1e6, 32.0, 4096.0, 0.0, 32.0)])
def test_rope_freqs(args):
    want = nm.rope_freqs(*args)
    got = np.full(args[0] // 2 + 1, -7.0)
    monet.call("monet_rope_freqs", got.ctypes.data, *args, *(1.0, 0.0, 0.0, 0.0)[len(args) - 2:])
    # a power of a 64-bit base: its exponent, at most ln(1e6) = 14 in size, carries 2^-52 relative; then three roundings
    assert np.abs(got[:-1] / want - 1).max() < 20 * 2.0 ** -52 and got[-1] == -7


def test_rope_freqs_refuses():
    a = np.zeros(4)
    at = a.ctypes.data
    refused("null", "monet_rope_freqs", None, 8, 1e4, 1.0, 0.0, 0.0, 0.0)
    for rot in (0, -2, 7, 514):
        refused("rot_dim", "monet_rope_freqs", at, rot, 1e4, 1.0, 0.0, 0.0, 0.0)
    for base in (0.0, -1.0, np.inf, np.nan):
        refused("base", "monet_rope_freqs", at, 8, base, 1.0, 0.0, 0.0, 0.0)
    for factor in (0.0, -1.0, np.inf, np.nan):
        refused("factor", "monet_rope_freqs", at, 8, 1e4, factor, 0.0, 0.0, 0.0)
    for blend in ((0.0, 1.0, 4.0), (8.0, 4.0, 4.0), (8.0, -1.0, 4.0), (np.nan, 1.0, 4.0), (8.0, 1.0, np.inf), (8.0, np.nan, 4.0)):
        refused("blend", "monet_rope_freqs", at, 8, 1e4, 1.0, *blend)


# ---------------------------------------------------------------------- refusals
def layernorm_args(**kw):
    a = dict(dtype=monet.BF16, param_dtype=monet.F32, dy=P, x=P, gamma=P, beta=P, y=P * 2, stats=P, dx=P * 2, dgamma=P, dbeta=P, rows=10, cols=64,
             dy_ld=64, x_ld=64, y_ld=64, dx_ld=64, eps=1e-5, accumulate=0, ws=P, ws_bytes=1 << 30)
    a.update(kw)
    fwd = [None] + [a[n] for n in "dtype param_dtype x gamma beta y stats rows cols x_ld y_ld eps".split()]
    bwd = [None] + [a[n] for n in "dtype param_dtype dy x gamma stats dx dgamma dbeta rows cols dy_ld x_ld dx_ld accumulate ws ws_bytes".split()]
    return fwd, bwd


@pytest.mark.parametrize("match,ways,kw", [
    ("dtype", "fb", dict(dtype=2)), ("param_dtype", "fb", dict(param_dtype=-1)), ("bad shape", "fb", dict(cols=0)), ("bad shape", "fb", dict(rows=-1)),
    ("too large", "fb", dict(rows=1 << 31)), ("too large", "fb", dict(cols=(1 << 20) + 1)), ("null", "fb", dict(x=None)), ("null", "f", dict(y=None)),
    ("null", "b", dict(dy=None)), ("aligned", "fb", dict(x=P + 1)), ("aligned", "fb", dict(x=P + 2, dtype=monet.F32)), ("aligned", "f", dict(y=P + 1)),
    ("aligned", "b", dict(dy=P + 1)), ("aligned", "b", dict(dx=P + 1)), ("aligned", "fb", dict(gamma=P + 2)), ("aligned", "f", dict(beta=P + 2)),
    ("aligned", "b", dict(dgamma=P + 2)), ("aligned", "b", dict(dbeta=P + 1, param_dtype=monet.BF16)), ("stats", "fb", dict(stats=P + 4)),
    ("stats", "b", dict(stats=None)), ("stride", "fb", dict(x_ld=63)), ("stride", "f", dict(y_ld=63)), ("stride", "b", dict(dy_ld=63)),
    ("stride", "b", dict(dx_ld=63)), ("stride", "fb", dict(x_ld=1 << 31)), ("in place", "f", dict(y=P, y_ld=65)), ("in place", "b", dict(dx=P, dx_ld=65)),
    ("eps", "f", dict(eps=0.0)), ("eps", "f", dict(eps=-1.0)), ("eps", "f", dict(eps=float("nan"))), ("accumulate", "b", dict(accumulate=8)),
    ("accumulate", "b", dict(accumulate=-1)), ("workspace", "b", dict(ws=None)), ("workspace", "b", dict(ws_bytes=64)), ("workspace", "b", dict(ws=P + 128)),
])
def test_layernorm_refuses(match, ways, kw):
    fwd, bwd = layernorm_args(**kw)
    if "f" in ways:
        refused(match, "monet_layernorm_fwd", *fwd)
    if "b" in ways:
        refused(match, "monet_layernorm_bwd", *bwd)


def test_layernorm_workspace_bytes():
    assert monet.call("monet_layernorm_bwd_workspace_bytes", monet.F32, 10, 64) > 0
    refused("dtype", "monet_layernorm_bwd_workspace_bytes", 7, 10, 64)
    refused("bad shape", "monet_layernorm_bwd_workspace_bytes", monet.F32, 10, 0)
    refused("too large", "monet_layernorm_bwd_workspace_bytes", monet.F32, 1 << 31, 64)


def rope_args(**kw):
    a = dict(dtype=monet.BF16, x=P, y=2 * P, positions=P, freqs=np.ones(256), tokens=10, heads=4, dim=64, rot=32, x_ld=256, y_ld=256, interleaved=0, scale=1.0,
             accumulate=0)
    a.update(kw)
    table = a["freqs"]
    a["freqs"] = None if table is None else table.ctypes.data
    return table, [None] + [a[n] for n in "dtype x y positions freqs tokens heads dim rot x_ld y_ld interleaved scale".split()], a["accumulate"]


@pytest.mark.parametrize("match,kw", [
    ("dtype", dict(dtype=5)), ("bad shape", dict(tokens=-1)), ("bad shape", dict(heads=0)), ("bad shape", dict(dim=0)), ("rot_dim", dict(rot=0)),
    ("rot_dim", dict(rot=33)), ("rot_dim", dict(rot=66)), ("rot_dim", dict(rot=514, dim=600, x_ld=2400, y_ld=2400)), ("too large", dict(tokens=1 << 24)),
    ("too large", dict(heads=1 << 20)), ("too large", dict(dim=1 << 24)), ("too large", dict(heads=1 << 30, dim=1 << 30)),
    ("scale", dict(scale=float("inf"))), ("scale", dict(scale=float("nan"))), ("null", dict(freqs=None)), ("null", dict(x=None)), ("null", dict(y=None)),
    ("frequencies", dict(freqs=np.full(256, np.nan))), ("frequencies", dict(freqs=np.full(256, np.inf))), ("aligned", dict(x=P + 1)),
    ("aligned", dict(y=P + 2, dtype=monet.F32)), ("aligned", dict(positions=P + 2)), ("stride", dict(x_ld=255)), ("stride", dict(y_ld=255)),
    ("stride", dict(x_ld=1 << 31)), ("in place", dict(y=P, y_ld=257)),
])
def test_rope_refuses(match, kw):
    keep, args, accumulate = rope_args(**kw)
    refused(match, "monet_rope_fwd", *args)
    refused(match, "monet_rope_bwd", *args, accumulate)


def test_rope_refuses_to_add_in_place():
    keep, args, _ = rope_args(y=P)
    refused("in place", "monet_rope_bwd", *args, 1)


def distill_args(**kw):
    a = dict(dtype=monet.BF16, x=P, w=P, index=P, target=P, target_lse=None, loss=P, lse=P, mass=P, delta=P, dx=P, dw=P, rows=10, width=64, vocab=1000, top=8,
             heat=2.0, accumulate=0, ws=P, ws_bytes=1 << 34)
    a.update(kw)
    fwd = [None] + [a[n] for n in "dtype x w index target target_lse loss lse mass delta rows width vocab top heat ws ws_bytes".split()]
    bwd = [None] + [a[n] for n in "dtype x w index lse mass delta dx dw rows width vocab top heat accumulate ws ws_bytes".split()]
    return fwd, bwd


@pytest.mark.parametrize("match,ways,kw", [
    ("dtype", "fb", dict(dtype=3)), ("bad shape", "fb", dict(rows=0)), ("bad shape", "fb", dict(width=0)), ("bad shape", "fb", dict(vocab=0)),
    ("entries", "fb", dict(top=0)), ("entries", "fb", dict(top=1025)), ("multiple of 8", "fb", dict(width=63)), ("too large", "fb", dict(rows=1 << 24)),
    ("temperature", "fb", dict(heat=0.0)), ("temperature", "fb", dict(heat=-1.0)), ("temperature", "fb", dict(heat=float("inf"))),
    ("temperature", "fb", dict(heat=float("nan"))), ("temperature", "fb", dict(heat=1e-45)), ("null", "fb", dict(x=None)), ("null", "fb", dict(w=None)),
    ("null", "fb", dict(index=None)), ("null", "f", dict(target=None)), ("null", "f", dict(loss=None)), ("null", "fb", dict(lse=None)),
    ("null", "fb", dict(mass=None)), ("null", "fb", dict(delta=None)), ("null", "b", dict(dx=None)), ("null", "b", dict(dw=None)),
    ("16-byte", "fb", dict(x=P + 8)), ("4-byte", "fb", dict(x=P + 2, dtype=monet.F32)), ("4-byte", "fb", dict(index=P + 2)),
    ("4-byte", "f", dict(target=P + 2)), ("4-byte", "f", dict(target_lse=P + 2)), ("4-byte", "fb", dict(delta=P + 1)), ("workspace", "fb", dict(ws=None)),
    ("workspace", "fb", dict(ws_bytes=64)), ("workspace", "fb", dict(ws=P + 16)),
])
def test_linear_distill_refuses(match, ways, kw):
    fwd, bwd = distill_args(**kw)
    if "f" in ways:
        refused(match, "monet_linear_distill_fwd", *fwd)
    if "b" in ways:
        refused(match, "monet_linear_distill_bwd", *bwd)


def test_linear_distill_workspace_bytes():
    need = lambda grad, *a: monet.call("monet_linear_distill_workspace_bytes", grad, *a)   # noqa: E731
    assert need(1, monet.BF16, 100, 64, 5000, 16) >= need(0, monet.BF16, 100, 64, 5000, 16) > 0
    refused("entries", "monet_linear_distill_workspace_bytes", 1, monet.BF16, 100, 64, 5000, 0)
    refused("multiple of 8", "monet_linear_distill_workspace_bytes", 1, monet.BF16, 100, 63, 5000, 4)
