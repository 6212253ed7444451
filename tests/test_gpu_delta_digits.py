"""Results of bfloat16 tensors come from products with all of float32's digits: sums that are what is left of far larger terms, and results that are roundings of
what float32 would give."""
import numpy as np
import pytest
import torch

import delta_util as O
from paper_2603_13810_amd import api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAMES = ("query", "key", "value", "gate", "write")
INF = float("inf")

# BASE and BASE + FINE: two bfloat16 numbers hold 1 and 2^-9 of either, which is all of the first and not the second.
FINE = 2.0 ** -18
BASE = 1.0 + 2.0 ** -9
# Every product and sum below is a whole number of FINE / 2 and smaller than 8, so that float32 holds it: exact, and one rounding of the terms' sum allowed.
# B, key heads, value heads, Dk, Dv; the last two take 32 columns of a state
SHAPES = [(1, 1, 1, 8, 5), (2, 1, 2, 40, 24), (1, 2, 2, 128, 40), (16, 8, 32, 24, 20), (8, 32, 64, 128, 33)]
PLACES = [0, 30, 65]           # the step that everything begins at, of 70


def still(B, hk, hv, dk, dv, T=70):
    """Steps that keep the state as it is and read nothing: open gates, nothing written, queries and keys of zero."""
    x = {n: torch.zeros(T, B, h, d) for n, h, d in (("query", hk, dk), ("key", hk, dk), ("value", hv, dv))}
    x["gate"], x["write"] = torch.full((T, B, hv), INF), torch.full((T, B, hv), -INF)
    return x


def signs(B, hv, dv):
    """1 and -1 in turn: FINE on either side."""
    s = torch.ones(B, hv, dv)
    s[..., 1::2] = -1
    s[:, 1::2] *= -1
    return s


def scan(x, h0, kept):
    x = {n: t.to(torch.bfloat16).to(DEV) for n, t in x.items()}
    return api.tac_delta_scan(*[x[n] for n in NAMES], h0=h0.to(DEV), want_kept=kept)


def close(got, want, terms):
    assert (np.abs(O.as64(got) - want.double().numpy()) <= terms * O.U).all(), float(np.abs(O.as64(got) - want.double().numpy()).max())


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("t0", PLACES)
@pytest.mark.parametrize("shape", SHAPES)
def test_outputs_from_states(shape, t0, kept):
    """out = (S_0 - S_1) / 2 of rows that are nearly the same."""
    B, hk, hv, dk, dv = shape
    x, fine = still(*shape), signs(B, hv, dv) * FINE
    h0 = torch.zeros(B, hv, dk, dv)
    h0[:, :, 0], h0[:, :, dk - 1] = BASE + fine, BASE
    x["query"][t0, ..., 0], x["query"][t0, ..., dk - 1] = 0.5, -0.5
    got = scan(x, h0, kept)
    close(got["out"][t0], fine / 2, 1.01)
    assert (got["out"][:t0] == 0).all() and (got["out"][t0 + 1:] == 0).all() and torch.equal(got["h_last"], h0.to(DEV))


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("t0", PLACES)
@pytest.mark.parametrize("shape", SHAPES)
def test_outputs_from_what_the_steps_write(shape, t0, kept):
    """Rows -2 (BASE + fine) and 2 BASE; each is halved by a step of its own, that writes BASE + fine and -BASE, and what is left of both is read: -fine."""
    B, hk, hv, dk, dv = shape
    x, fine = still(*shape), signs(B, hv, dv) * FINE
    h0 = torch.zeros(B, hv, dk, dv)
    h0[:, :, 1], h0[:, :, 4] = -2 * (BASE + fine), 2 * BASE
    x["key"][t0, ..., 1], x["key"][t0 + 1, ..., 4] = 1, 1
    x["write"][t0:t0 + 2] = 0
    x["query"][t0 + 1, ..., 1], x["query"][t0 + 1, ..., 4] = 1, 1
    got = scan(x, h0, kept)
    close(got["out"][t0 + 1], -fine, 6.02)
    close(got["h_last"][:, :, 1], -(BASE + fine), 0)
    if kept:
        close(got["updates"][t0], BASE + fine, 0)


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("t0", PLACES)
@pytest.mark.parametrize("shape", SHAPES)
def test_outputs_from_products_of_queries_and_keys(shape, t0, kept):
    """Two steps write 1 and -1 under keys whose products with the query are BASE + FINE and BASE."""
    B, hk, hv, dk, dv = shape
    x, sign = still(*shape), signs(B, hv, dv)
    x["key"][t0, ..., 0:3] = 1
    x["key"][t0 + 1, ..., 3:5] = 1
    x["value"][t0], x["value"][t0 + 1] = 2 * sign, -2 * sign
    x["write"][t0:t0 + 2] = 0
    x["query"][t0 + 1, ..., :5] = torch.tensor([1, 2.0 ** -9, FINE, 1, 2.0 ** -9])
    got = scan(x, torch.zeros(B, hv, dk, dv), kept)
    close(got["out"][t0 + 1], sign * FINE, 2.01)


def between(name, got, want, bound):
    """got is the rounding of a number that is at most `bound` from what is wanted."""
    ends = [torch.from_numpy(want + s * bound).to(got.dtype).double().numpy() for s in (-1, 1)]
    off = np.maximum(ends[0] - O.as64(got), O.as64(got) - ends[1])
    assert (off <= 0).all(), (name, int((off > 0).sum()), off.size)


# As for float32 tensors: sums over up to 128 features and 64 steps of products with a relative error of 2^-24 or so, of numbers that come from two or three such
# sums: 4 sqrt(192) independent roundings in the 2-norm, four times as many, by the root mean square, in the worst of some 10^5 results.
NORM, WORST = 64 * O.U, 256 * O.U


def plain_bound(want):
    return WORST * (np.abs(want) + np.sqrt((want * want).mean()))


@pytest.mark.parametrize("T,B,hk,hv,dk,dv", [(130, 2, 2, 4, 64, 64), (260, 1, 2, 2, 128, 128), (100, 3, 1, 2, 33, 70)])
def test_outputs_are_roundings_of_float32(T, B, hk, hv, dk, dv):
    x, h0 = O.delta_inputs(T, B, hk, hv, dk, dv, torch.bfloat16, 40 + dk)
    got = api.tac_delta_scan(*[x[n] for n in NAMES], h0=h0)
    out, S, _ = O.delta(*[O.as64(x[n]) for n in NAMES], h0=O.as64(h0))
    between("out", got["out"], out, plain_bound(out))


# ---- gradients -----------------------------------------------------------------------------------

GRADS = ("grad_query", "grad_key", "grad_value", "grad_gate", "grad_write", "grad_h0")


def backward(x, h0, grad_out=None, grad_last=None):
    x = {n: t.to(torch.bfloat16).to(DEV) for n, t in x.items()}
    args = [x[n] for n in NAMES]
    got = api.tac_delta_scan(*args, h0=h0.to(DEV), want_kept=True)
    grad_out = torch.zeros_like(x["value"]) if grad_out is None else grad_out.to(torch.bfloat16).to(DEV)
    return got, api.tac_delta_scan_backward(*args, got["states"], got["updates"], grad_out, grad_h_last=None if grad_last is None else grad_last.to(DEV))


def by_head(B, hk, hv, dk):
    """1 and -1 in turn, one for all heads of values that share a head of keys, and one for every feature of a key; how many share one."""
    heads, features = torch.ones(B, hk, 1), torch.ones(dk)
    heads[:, 1::2] = -1
    features[1::2] = -1
    return heads, heads.repeat_interleave(hv // hk, 1), features, hv // hk


@pytest.mark.parametrize("t0", PLACES)
@pytest.mark.parametrize("shape", SHAPES)
def test_query_gradients_from_states(shape, t0):
    """grad_query = S grad_out, of two columns that are nearly the same."""
    B, hk, hv, dk, dv = shape
    key_heads, heads, features, share = by_head(B, hk, hv, dk)
    x, h0, go = still(*shape), torch.zeros(B, hv, dk, dv), torch.zeros(70, B, hv, dv)
    h0[..., 0], h0[..., dv - 1] = BASE + heads * features * FINE, BASE
    go[t0, ..., 0], go[t0, ..., dv - 1] = 0.5, -0.5
    _, got = backward(x, h0, go)
    close(got["grad_query"][t0], share * key_heads * features * FINE / 2, 1.01 * share)


@pytest.mark.parametrize("t0", PLACES)
@pytest.mark.parametrize("shape", SHAPES)
def test_key_gradients_from_the_states_gradients(shape, t0):
    """A step that writes 1 and -1 into two columns of a state whose gradients are nearly the same."""
    B, hk, hv, dk, dv = shape
    key_heads, heads, features, share = by_head(B, hk, hv, dk)
    x, last = still(*shape), torch.zeros(B, hv, dk, dv)
    last[..., 0], last[..., dv - 1] = BASE + heads * features * FINE, BASE
    x["value"][t0, ..., 0], x["value"][t0, ..., dv - 1] = 1, -1
    x["write"][t0] = INF
    _, got = backward(x, torch.zeros_like(last), grad_last=last)
    close(got["grad_key"][t0], share * key_heads * features * FINE, 2.01 * share)


@pytest.mark.parametrize("t0", PLACES)
@pytest.mark.parametrize("shape", SHAPES)
def test_key_gradients_from_what_a_step_writes(shape, t0):
    """A step halves a row and writes BASE + fine and BASE, into columns whose gradients are 1 and -1."""
    B, hk, hv, dk, dv = shape
    key_heads, heads, features, share = by_head(B, hk, hv, dk)
    x, h0, last = still(*shape), torch.zeros(B, hv, dk, dv), torch.zeros(B, hv, dk, dv)
    h0[:, :, 1, 0], h0[:, :, 1, dv - 1] = -2 * (BASE + heads[..., 0] * FINE), -2 * BASE
    last[..., 0], last[..., dv - 1] = features, -features
    last[:, :, 1] = 0
    x["key"][t0, ..., 1] = 1
    x["write"][t0] = 0
    kept, got = backward(x, h0, grad_last=last)
    want = share * key_heads * features * FINE
    want[..., 1] = 0
    close(kept["updates"][t0, ..., 0], BASE + heads[..., 0] * FINE, 0)
    close(got["grad_key"][t0], want, 2.01 * share)


@pytest.mark.parametrize("digits", ["gradients", "states"])
@pytest.mark.parametrize("t0", PLACES)
@pytest.mark.parametrize("shape", SHAPES)
def test_key_gradients_from_what_a_step_reads(shape, t0, digits):
    """-b S r, where r = dS^T key is BASE + fine and BASE and a row of S is 1 and -1, or the other way around."""
    B, hk, hv, dk, dv = shape
    key_heads, heads, features, share = by_head(B, hk, hv, dk)
    x, h0, last = still(*shape), torch.zeros(B, hv, dk, dv), torch.zeros(B, hv, dk, dv)
    if digits == "gradients":
        last[:, :, 1, 0], last[:, :, 1, dv - 1] = BASE + heads[..., 0] * FINE, BASE
        h0[..., 0], h0[..., dv - 1] = features, -features
    else:
        last[:, :, 1, 0], last[:, :, 1, dv - 1] = 1, -1
        h0[..., 0], h0[..., dv - 1] = BASE + heads * features * FINE, BASE
    h0[:, :, 1] = 0
    x["key"][t0, ..., 1] = 1
    x["write"][t0] = 0
    _, got = backward(x, h0, grad_last=last)
    want = -share * key_heads * features * FINE / 2
    want[..., 1] = 0
    close(got["grad_key"][t0], want, 1.01 * share)


def two_writers(shape, t0):
    """Two steps that write BASE + fine and -BASE into feature 2, whose keys have it in common."""
    B, hk, hv, dk, dv = shape
    key_heads, heads, _, share = by_head(B, hk, hv, dk)
    x, h0, fine = still(*shape), torch.zeros(B, hv, dk, dv), heads * FINE
    h0[:, :, 0], h0[:, :, 1] = -2 * (BASE + fine), BASE - fine
    x["key"][t0, ..., 0], x["key"][t0, ..., 2] = 1, 1
    x["key"][t0 + 1, ..., 1], x["key"][t0 + 1, ..., 2] = 1, 1
    x["write"][t0:t0 + 2] = 0
    return x, h0, share * key_heads[..., 0] * FINE, share


@pytest.mark.parametrize("t0", PLACES)
@pytest.mark.parametrize("shape", SHAPES)
def test_query_gradients_from_products_of_gradients_and_updates(shape, t0):
    B, hk, hv, dk, dv = shape
    x, h0, fine, share = two_writers(shape, t0)
    go = torch.zeros(70, B, hv, dv)
    go[t0 + 1, ..., 3] = 1
    kept, got = backward(x, h0, go)
    assert (kept["updates"][t0 + 1] == -BASE).all()
    close(got["grad_query"][t0 + 1, ..., 2], fine, 2.01 * share)


@pytest.mark.parametrize("t0", PLACES)
@pytest.mark.parametrize("shape", SHAPES)
def test_key_gradients_from_products_of_gradients_and_updates(shape, t0):
    """A third step reads what the two wrote, -S r / 2."""
    B, hk, hv, dk, dv = shape
    x, h0, fine, share = two_writers(shape, t0)
    x["key"][t0 + 2, ..., 3] = 1
    x["write"][t0 + 2] = 0
    last = torch.zeros(B, hv, dk, dv)
    last[:, :, 3, 3] = 1
    _, got = backward(x, h0, grad_last=last)
    close(got["grad_key"][t0 + 2, ..., 2], -fine / 2, 1.01 * share)


@pytest.mark.parametrize("t0", PLACES)
@pytest.mark.parametrize("shape", SHAPES)
def test_key_gradients_from_later_queries(shape, t0):
    """A step writes BASE + fine and BASE into two columns; two queries read them, with opposite signs."""
    B, hk, hv, dk, dv = shape
    key_heads, heads, _, share = by_head(B, hk, hv, dk)
    x, h0, go = still(*shape), torch.zeros(B, hv, dk, dv), torch.zeros(70, B, hv, dv)
    h0[:, :, 0, 0], h0[:, :, 0, dv - 1] = -2 * (BASE + heads[..., 0] * FINE), -2 * BASE
    x["key"][t0, ..., 0] = 1
    x["write"][t0] = 0
    x["query"][t0 + 1, ..., 2], x["query"][t0 + 2, ..., 2] = 1, -1
    go[t0 + 1, ..., 0], go[t0 + 2, ..., dv - 1] = 1, 1
    _, got = backward(x, h0, go)
    close(got["grad_key"][t0, ..., 2], share * key_heads[..., 0] * FINE, 2.01 * share)


@pytest.mark.parametrize("T,B,hk,hv,dk,dv", [(130, 2, 2, 4, 64, 64), (260, 1, 2, 2, 128, 128), (100, 3, 1, 2, 33, 70)])
def test_gradients_are_roundings_of_float32(T, B, hk, hv, dk, dv):
    x, h0 = O.delta_inputs(T, B, hk, hv, dk, dv, torch.bfloat16, 50 + dk)
    g = torch.Generator().manual_seed(dk)
    go, last = torch.randn(T, B, hv, dv, generator=g), torch.randn(B, hv, dk, dv, generator=g)
    _, got = backward(x, h0, go, last)
    args = [O.as64(x[n]) for n in NAMES]
    kept = O.delta(*args, h0=O.as64(h0))[2]
    want, sizes = O.delta_backward(*args, kept, O.as64(go.to(torch.bfloat16)), grad_last=O.as64(last))
    for name, w in zip(GRADS[:5], want):
        between(name, got[name], w, NORM * sizes if name == "grad_gate" else plain_bound(w))
