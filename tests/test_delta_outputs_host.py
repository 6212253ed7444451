"""Calls whose outputs begin where an input or another output does, without a GPU: all are refused before anything is launched."""
import pytest

from paper_2603_13810_amd import api
from test_delta_host import P, delta_desc, scan

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
