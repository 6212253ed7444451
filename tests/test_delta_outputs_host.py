"""Calls whose outputs begin where an input or another output does, without a GPU: all are refused before anything is launched."""
import ctypes

import pytest

from paper_2603_13810_amd import api
from test_delta_host import P, delta_desc, head_norm, head_norm_backward, heads_desc, scan, scan_backward, step

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


STEP = ("query", "key", "value", "gate", "write", "pool", None, "slots", "out")


@pytest.mark.parametrize("written", ["pool", "out"])
def test_delta_step(written):
    w = STEP.index(written)
    apart = {i: APART[i] for i, n in enumerate(STEP) if n}
    for i, other in enumerate(STEP):
        if other not in (None, written):
            assert step(delta_desc(T=1), {**apart, w: APART[i]}) == api.TAC_ERR_BAD_PARAM, other


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


# What is ignored.  Every call is refused by the last of the checks, queries (or their gradients) in place with other strides: all others have passed.
ODD = P + 1


def in_place(d, key=None, gain_key=None, positions=None, out_key=None):
    return api.lib().tac_head_norm(ctypes.byref(d), APART[0], key, APART[1], gain_key, positions, APART[0], out_key, None)


def in_place_backward(d, key=None, gain_key=None, positions=None, grad_out_key=None, grad_key=None, grad_gain_query=None, grad_gain_key=None, workspace=None):
    return api.lib().tac_head_norm_backward(ctypes.byref(d), APART[0], key, APART[1], gain_key, positions, APART[2], grad_out_key, APART[2], grad_key, grad_gain_query,
                                            grad_gain_key, workspace, None)


NO_KEYS = dict(key_heads=0, key=(0, 0), out_key=(-1, 7), grad_key=(3, 3))


@pytest.mark.parametrize("at", [None, ODD])
def test_without_keys_nothing_of_them_counts(at):
    assert in_place(heads_desc(out_query=(128, 16), **NO_KEYS), key=at, gain_key=at, out_key=at, positions=APART[3]) == api.TAC_ERR_BAD_PARAM
    assert in_place_backward(heads_desc(grad_query=(128, 16), **NO_KEYS), key=at, gain_key=at, grad_out_key=at, grad_key=at, grad_gain_key=at,
                             positions=APART[3]) == api.TAC_ERR_BAD_PARAM


@pytest.mark.parametrize("at", [None, ODD])
def test_without_a_rotation_no_position_counts(at):
    for base in (0.0, float("nan")):
        assert in_place(heads_desc(out_query=(128, 16), axes=0, base=base, pairs=(0, -1, 99, 1 << 30), **NO_KEYS), positions=at) == api.TAC_ERR_BAD_PARAM
        assert in_place_backward(heads_desc(grad_query=(128, 16), axes=0, base=base, **NO_KEYS), positions=at) == api.TAC_ERR_BAD_PARAM


@pytest.mark.parametrize("at", [None, P + 8])
def test_without_a_gains_gradient_no_workspace_counts(at):
    assert in_place_backward(heads_desc(grad_query=(128, 16)), key=APART[4], gain_key=APART[5], positions=APART[3], grad_out_key=APART[6], grad_key=APART[7],
                             workspace=at) == api.TAC_ERR_BAD_PARAM


def test_what_is_missing_otherwise():
    """The same calls with keys, a rotation and a gain's gradient."""
    assert in_place(heads_desc(out_query=(128, 16)), positions=APART[3]) == api.TAC_ERR_NULL
    assert in_place(heads_desc(out_query=(128, 16), **NO_KEYS)) == api.TAC_ERR_NULL
    assert in_place_backward(heads_desc(grad_query=(128, 16), **NO_KEYS), positions=APART[3], grad_gain_query=APART[4]) == api.TAC_ERR_NULL
    assert in_place_backward(heads_desc(grad_query=(128, 16), **NO_KEYS), positions=APART[3], grad_gain_query=APART[4], workspace=P + 8) == api.TAC_ERR_ALIGN
