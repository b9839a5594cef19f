"""Calls that the transformer operators refuse before anything is enqueued, which needs no GPU: the addresses are never read."""
import pytest

from paper_2010_14501_amd import monet

P = 1 << 20


def test_linear_ce_refuses_large_products_before_its_first_launch():
    rows, width = (1 << 24) - 1, 1 << 20
    with pytest.raises(monet.MonetError, match="too large"):
        monet.call("monet_linear_ce_workspace_bytes", 1, monet.BF16, rows, width, 64)
    with pytest.raises(monet.MonetError, match="too large"):
        monet.call("monet_linear_ce_bwd", None, monet.BF16, P, P, P, P, P, P, rows, width, 64, 0, P, 1 << 60)
    # rows x width tiles of 256: 2^23 are too many, a row less of them is not
    assert monet.call("monet_linear_ce_workspace_bytes", 1, monet.BF16, ((1 << 15) - 1) * 256, 1 << 16, 64) > 0
    with pytest.raises(monet.MonetError, match="too large"):
        monet.call("monet_linear_ce_workspace_bytes", 1, monet.BF16, (1 << 15) * 256, 1 << 16, 64)


def test_act8_wgrad_refuses_large_results_before_its_first_launch():
    for cols, outs in ((1 << 22, 1 << 22), (1 << 24, 1 << 24)):          # through the workspace, and directly
        with pytest.raises(monet.MonetError, match="too large"):
            monet.call("monet_act8_wgrad_workspace_bytes", monet.BF16, 64, cols, outs)
        with pytest.raises(monet.MonetError, match="too large"):
            monet.call("monet_act8_wgrad", None, monet.BF16, P, P, P, 64, cols, outs, P, 1 << 60)


@pytest.mark.parametrize("name", ["lse", "cu"])
def test_attention_refuses_numbers_off_their_alignment(name):
    a = dict(lse=P, cu=P)
    a[name] = P + 2
    shape = (a["cu"], 3, 100, 8, 4, 64, 512, 256, 256, 512, 0.125)
    with pytest.raises(monet.MonetError, match="4-byte aligned"):
        monet.call("monet_attention_fwd", None, monet.BF16, P, P, P, P, a["lse"], *shape)
    with pytest.raises(monet.MonetError, match="4-byte aligned"):
        monet.call("monet_attention_bwd", None, monet.BF16, P, P, P, P, P, a["lse"], P, P, P, *shape, 0, P, 1 << 30)


@pytest.mark.parametrize("name", ["labels", "loss", "lse", "x"])
def test_linear_ce_refuses_numbers_off_their_alignment(name):
    a = dict(labels=P, loss=P, lse=P, x=P)
    a[name] = P + 1
    with pytest.raises(monet.MonetError, match="4-byte aligned"):
        monet.call("monet_linear_ce_fwd", None, monet.F32, a["x"], P, a["labels"], a["loss"], a["lse"], 50, 64, 1000, P, 1 << 30)
    if name != "loss":
        with pytest.raises(monet.MonetError, match="4-byte aligned"):
            monet.call("monet_linear_ce_bwd", None, monet.F32, a["x"], P, a["labels"], a["lse"], P, P, 50, 64, 1000, 0, P, 1 << 30)


@pytest.mark.parametrize("heads,kv_heads,dim,tokens", [(4, 1, 64, 12000), (8, 1, 64, 4000), (16, 4, 128, 6000), (32, 8, 128, 5000)])
def test_empty_sequences_take_no_ranges_from_a_long_one(heads, kv_heads, dim, tokens):
    """The way along the rows behind a key is cut into ranges whose sums the workspace holds.  Offsets that are padded with empty sequences must not
    make the same tokens go uncut: no fewer ranges in fp32, and two at least in bf16."""
    sums = 2 * tokens * kv_heads * dim * 4
    need = lambda dtype, seqs: monet.call("monet_attention_bwd_workspace_bytes", dtype, seqs, tokens, heads, kv_heads, dim)   # noqa: E731
    for seqs in (1, 10, 64, 256):
        assert need(monet.F32, seqs) == need(monet.F32, 1) > 2 * sums
        assert need(monet.BF16, seqs) > 2 * sums


def test_act8_bytes_refuses_what_pack_refuses():
    """2^35 codes are more than a launch takes; one row fewer is not."""
    rows, cols = 1 << 11, 1 << 24
    with pytest.raises(monet.MonetError, match="too many"):
        monet.call("monet_act8_pack", None, monet.BF16, P, cols, P, rows, cols)
    with pytest.raises(monet.MonetError, match="too many"):
        monet.call("monet_act8_bytes", rows, cols)
    assert monet.call("monet_act8_bytes", rows - 1, cols) == (rows - 1) * cols // 32 * 33
