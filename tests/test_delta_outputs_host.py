"""Calls whose outputs begin where an input or another output does, without a GPU: all are refused before anything is launched."""
import pytest

from paper_2603_13810_amd import api
from test_delta_host import P, delta_desc, head_norm, head_norm_backward, scan, scan_backward

APART = [P + 4096 * (i + 1) for i in range(24)]


def at(n, **moved):
    """Addresses that have nothing in common, but for the one that is moved."""
    return {**{i: APART[i] for i in range(n)}, **{int(i[1:]): a for i, a in moved.items()}}


SCAN = ("query", "key", "value", "gate", "write", "lengths", "h0", "out", "h_last", "states", "updates", "workspace")


@pytest.mark.parametrize("written", ["out", "h_last", "states", "updates", "workspace"])
def test_delta_scan(written):
    w = SCAN.index(written)
    for other in SCAN:
        if other == written or {written, other} == {"h_last", "h0"}:       # the last states may take the first ones' place
            continue
        assert scan(delta_desc(), at(12, **{"_%d" % w: APART[SCAN.index(other)]})) == api.TAC_ERR_BAD_PARAM, other
    # also where nothing is kept for the backward pass
    for other in SCAN[:6]:
        if written in ("out", "h_last", "workspace"):
            assert scan(delta_desc(), {**at(12, **{"_%d" % w: APART[SCAN.index(other)]}), 9: None, 10: None}) == api.TAC_ERR_BAD_PARAM, other


BACK = ("query", "key", "value", "gate", "write", "lengths", "states", "updates", "grad_out", "grad_h_last", "grad_query", "grad_key", "grad_value", "grad_gate", "grad_write", "grad_h0",
        "workspace")


@pytest.mark.parametrize("written", BACK[10:])
def test_delta_scan_backward(written):
    w = BACK.index(written)
    for other in BACK:
        if other == written or {written, other} == {"grad_h0", "grad_h_last"}:
            continue
        assert scan_backward(delta_desc(), at(17, **{"_%d" % w: APART[BACK.index(other)]})) == api.TAC_ERR_BAD_PARAM, other


HEADS_BACK = ("query", "key", "gain_query", "gain_key", "positions", "grad_out_query", "grad_out_key", "grad_query_at", "grad_key_at", "grad_gain_query", "grad_gain_key", "workspace")


@pytest.mark.parametrize("written", HEADS_BACK[9:])
def test_gradients_of_gains(written):
    apart = dict(zip(HEADS_BACK, APART))
    for other in HEADS_BACK:
        if other != written:
            assert head_norm_backward(**{**apart, written: apart[other]}) == api.TAC_ERR_BAD_PARAM, other


HEADS = ("query", "key", "gain_query", "gain_key", "positions", "out_query", "out_key")


@pytest.mark.parametrize("written", ["out_query", "out_key"])
def test_head_norm(written):
    apart = dict(zip(HEADS, APART))
    for other in HEADS:
        if other not in (written, written[4:]):                            # heads in place
            assert head_norm(**{**apart, written: apart[other]}) == api.TAC_ERR_BAD_PARAM, other


@pytest.mark.parametrize("written", ["grad_query_at", "grad_key_at"])
def test_head_norm_backward(written):
    apart = dict(zip(HEADS_BACK, APART))
    for other in HEADS_BACK:
        if other not in (written, "grad_out_" + written[5:-3]):
            assert head_norm_backward(**{**apart, written: apart[other]}) == api.TAC_ERR_BAD_PARAM, other
