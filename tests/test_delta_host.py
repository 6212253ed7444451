"""Head norm and gated delta rule, without a GPU: struct layouts, sizes, refusals before anything is launched."""
import ctypes
import os
import re

import pytest

from paper_2603_13810_amd import api

HEADER = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "tac.h")).read()
P, ODD = 1 << 20, (1 << 20) + 1              # addresses that are never read: nothing is launched


def fields_of(name):
    body = HEADER[HEADER.index("typedef struct %s {" % name[:-2]):HEADER.index("} %s;" % name)]
    body = re.sub(r"/\*.*?\*/", "", body[body.index("{") + 1:], flags=re.S)
    kinds = {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float, "double": ctypes.c_double,
             "tac_head_strides_t": api.tac_head_strides_t, "tac_delta_strides_t": api.tac_delta_strides_t}
    out = []
    for kind, names in re.findall(r"(\w+)\s+([^;]+);", body):
        for n in names.split(","):
            m = re.match(r"\s*(\w+)(?:\[(\w+)\])?\s*$", n)
            out.append((m.group(1), kinds[kind] * getattr(api, m.group(2)) if m.group(2) else kinds[kind]))
    return out


@pytest.mark.parametrize("struct", [api.tac_head_strides_t, api.tac_head_norm_desc_t, api.tac_delta_strides_t, api.tac_delta_desc_t])
def test_struct_layouts_match_the_header(struct):
    assert fields_of(struct.__name__) == list(struct._fields_)


def test_constants_match_the_header():
    for n in ("TAC_ROTATION_AXES", "TAC_HEAD_MAX_FEATURES", "TAC_DELTA_CHUNK", "TAC_DELTA_MAX_KEY", "TAC_DELTA_MAX_VALUE"):
        assert int(re.search(r"#define %s (\d+)" % n, HEADER).group(1)) == getattr(api, n)


def heads_desc(**kw):
    s = api.tac_head_strides_t
    d = dict(rows=5, query_heads=4, key_heads=2, D=16, dtype=api.TAC_BF16, axes=2, interleaved=0, eps=1e-6, base=10000.0)
    for n, heads in (("query", 4), ("key", 2), ("out_query", 4), ("out_key", 2), ("grad_query", 4), ("grad_key", 2)):
        d[n] = kw.pop(n, (heads * 16, 16))
    pairs = kw.pop("pairs", (3, 5, 0, 0))
    d.update(kw)
    d = {k: s(*v) if isinstance(v, tuple) else v for k, v in d.items()}
    return api.tac_head_norm_desc_t(pairs=(ctypes.c_int32 * 4)(*pairs), **d)


def head_norm(desc=True, query=P, key=P, gain_query=P, gain_key=P, positions=P, out_query=P, out_key=P, **kw):
    return api.lib().tac_head_norm(ctypes.byref(heads_desc(**kw)) if desc else None, query, key, gain_query, gain_key, positions, out_query, out_key, None)


def head_norm_backward(desc=True, query=P, key=P, gain_query=P, gain_key=P, positions=P, grad_out_query=P, grad_out_key=P, grad_query_at=P, grad_key_at=P,
                       grad_gain_query=P, grad_gain_key=P, workspace=P, **kw):
    return api.lib().tac_head_norm_backward(ctypes.byref(heads_desc(**kw)) if desc else None, query, key, gain_query, gain_key, positions, grad_out_query,
                                            grad_out_key, grad_query_at, grad_key_at, grad_gain_query, grad_gain_key, workspace, None)


COMMON = [
    (dict(desc=False), "NULL"), (dict(query=None), "NULL"), (dict(key=None), "NULL"), (dict(positions=None), "NULL"),
    (dict(rows=0), "BAD_SHAPE"), (dict(rows=1 << 31), "BAD_SHAPE"), (dict(query_heads=0), "BAD_SHAPE"), (dict(key_heads=-1), "BAD_SHAPE"),
    (dict(D=15), "BAD_SHAPE"), (dict(D=0), "BAD_SHAPE"), (dict(query=(64, 15)), "BAD_SHAPE"), (dict(query=(15, 16)), "BAD_SHAPE"), (dict(key=(1 << 60, 16)), "BAD_SHAPE"),
    (dict(out_key=(32, 0)), "BAD_SHAPE"), (dict(query_heads=65535, key_heads=1), "BAD_SHAPE"),
    (dict(dtype=2), "BAD_PARAM"), (dict(eps=-1.0), "BAD_PARAM"), (dict(eps=float("nan")), "BAD_PARAM"), (dict(eps=float("inf")), "BAD_PARAM"), (dict(axes=5), "BAD_PARAM"),
    (dict(axes=-1), "BAD_PARAM"), (dict(pairs=(4, 5, 0, 0)), "BAD_PARAM"), (dict(pairs=(0, 5, 0, 0)), "BAD_PARAM"), (dict(pairs=((1 << 31) - 1, (1 << 31) - 1, 0, 0)), "BAD_PARAM"),
    (dict(base=0.0), "BAD_PARAM"), (dict(base=float("inf")), "BAD_PARAM"), (dict(base=float("nan")), "BAD_PARAM"),
    (dict(D=514, query=(5000, 514), key=(5000, 514), out_query=(5000, 514), out_key=(5000, 514), grad_query=(5000, 514), grad_key=(5000, 514)), "UNSUPPORTED"),
    (dict(gain_query=P + 2), "ALIGN"), (dict(positions=P + 2), "ALIGN")]


@pytest.mark.parametrize("kw,status", COMMON + [(dict(out_query=ODD), "ALIGN")])
def test_head_norm_refuses(kw, status):
    # tensors and their strides have the same names here: addresses are whole numbers
    if isinstance(kw.get("query"), tuple) or isinstance(kw.get("key"), tuple) or isinstance(kw.get("out_key"), tuple):
        kw = dict(kw)
        d = heads_desc(**kw)
        assert api.lib().tac_head_norm(ctypes.byref(d), P, P, P, P, P, P, P, None) == getattr(api, "TAC_ERR_" + status)
        assert api.lib().tac_head_norm_backward(ctypes.byref(d), P, P, P, P, P, P, P, P, P, P, P, P, None) == getattr(api, "TAC_ERR_" + status)
        return
    if "out_query" in kw:
        assert api.lib().tac_head_norm(ctypes.byref(heads_desc()), P, P, P, P, P, kw["out_query"], P, None) == getattr(api, "TAC_ERR_" + status)
        return
    assert head_norm(**kw) == getattr(api, "TAC_ERR_" + status)
    assert head_norm_backward(**kw) == getattr(api, "TAC_ERR_" + status)


@pytest.mark.parametrize("kw,status", [(dict(grad_out_query=None), "NULL"), (dict(grad_out_key=None), "NULL"), (dict(grad_query_at=None), "NULL"), (dict(grad_key_at=None), "NULL"),
                                       (dict(workspace=None), "NULL"), (dict(workspace=P + 8), "ALIGN"), (dict(grad_gain_key=P + 2), "ALIGN"), (dict(grad_query_at=ODD), "ALIGN")])
def test_head_norm_backward_refuses(kw, status):
    assert head_norm_backward(**kw) == getattr(api, "TAC_ERR_" + status)


def test_head_norm_refuses_outputs_on_other_tensors():
    a = [P + 4096 * i for i in range(8)]
    f = dict(query=a[0], key=a[1], out_query=a[2], out_key=a[3])
    for kw in (dict(out_query=a[1]), dict(out_key=a[0]), dict(out_key=a[2])):
        assert head_norm(**{**f, **kw}) == api.TAC_ERR_BAD_PARAM
    b = dict(query=a[0], key=a[1], grad_out_query=a[2], grad_out_key=a[3], grad_query_at=a[4], grad_key_at=a[5])
    for kw in (dict(grad_query_at=a[0]), dict(grad_query_at=a[1]), dict(grad_query_at=a[3]), dict(grad_key_at=a[0]), dict(grad_key_at=a[1]), dict(grad_key_at=a[2]), dict(grad_key_at=a[4])):
        assert head_norm_backward(**{**b, **kw}) == api.TAC_ERR_BAD_PARAM
    call = lambda d, q, k, oq, ok: api.lib().tac_head_norm(ctypes.byref(d), q, k, P, P, P, oq, ok, None)
    assert call(heads_desc(out_query=(128, 16)), a[0], a[1], a[0], a[3]) == api.TAC_ERR_BAD_PARAM          # in place with other strides
    assert call(heads_desc(out_key=(16, 80)), a[0], a[1], a[2], a[1]) == api.TAC_ERR_BAD_PARAM
    back = lambda d, gq, gk: api.lib().tac_head_norm_backward(ctypes.byref(d), a[0], a[1], P, P, P, a[2], a[3], gq, gk, P, P, P, None)
    assert back(heads_desc(grad_query=(128, 16)), a[2], a[5]) == api.TAC_ERR_BAD_PARAM
    assert back(heads_desc(grad_key=(16, 80)), a[4], a[3]) == api.TAC_ERR_BAD_PARAM


def test_what_is_ignored_may_be_anything():
    """No keys, no rotation, no gain's gradient: their pointers and sizes do not count.  Refused by the features alone, so that nothing is launched."""
    bad = dict(D=15)
    assert head_norm(key_heads=0, key=None, **bad) == api.TAC_ERR_BAD_SHAPE
    assert api.lib().tac_head_norm_workspace_bytes(ctypes.byref(heads_desc(D=15))) == 0
    assert api.lib().tac_head_norm_workspace_bytes(ctypes.byref(heads_desc())) > 0


def delta_desc(**kw):
    s = api.tac_delta_strides_t
    B, hk, hv, dk, dv = 3, 2, 4, 8, 6
    d = dict(T=7, B=B, k_heads=hk, v_heads=hv, Dk=dk, Dv=dv, dtype=api.TAC_BF16)
    for n in ("query", "key", "grad_query", "grad_key"):
        d[n] = (B * hk * dk, hk * dk, dk)
    for n in ("value", "out", "grad_value"):
        d[n] = (B * hv * dv, hv * dv, dv)
    for n in ("gate", "write", "grad_gate", "grad_write"):
        d[n] = (B * hv, hv, 1)
    d.update(kw)
    return api.tac_delta_desc_t(**{k: s(*v) if isinstance(v, tuple) else v for k, v in d.items()})


def scan(desc, at=None):
    a = [P] * 12
    for i, v in (at or {}).items():
        a[i] = v
    return api.lib().tac_delta_scan(ctypes.byref(desc) if desc else None, *a, None)


def scan_backward(desc, at=None):
    a = [P] * 17
    for i, v in (at or {}).items():
        a[i] = v
    return api.lib().tac_delta_scan_backward(ctypes.byref(desc) if desc else None, *a, None)


def step(desc, at=None, n_slots=9):
    a = [P, P, P, P, P, P, n_slots, P, P]
    for i, v in (at or {}).items():
        a[i] = v
    return api.lib().tac_delta_step(ctypes.byref(desc) if desc else None, *a, None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=0), "BAD_SHAPE"), (dict(T=1 << 31), "BAD_SHAPE"), (dict(B=0), "BAD_SHAPE"), (dict(k_heads=0), "BAD_SHAPE"), (dict(v_heads=3), "BAD_SHAPE"), (dict(v_heads=0), "BAD_SHAPE"),
    (dict(Dk=0), "BAD_SHAPE"), (dict(Dv=0), "BAD_SHAPE"), (dict(Dk=129), "UNSUPPORTED"), (dict(Dv=4097), "UNSUPPORTED"), (dict(dtype=2), "BAD_PARAM"),
    (dict(B=1 << 30, v_heads=2), "BAD_SHAPE"), (dict(T=(1 << 31) - 1), "BAD_SHAPE"),
    (dict(query=(48, 16, 7)), "BAD_SHAPE"), (dict(key=(48, 7, 8)), "BAD_SHAPE"), (dict(value=(5, 24, 6)), "BAD_SHAPE"), (dict(value=(72, 24, -6)), "BAD_SHAPE"),
    (dict(gate=(12, 4, 2)), "BAD_SHAPE"), (dict(write=(12, 3, 1)), "BAD_SHAPE"), (dict(out=(0, 24, 6)), "BAD_SHAPE"), (dict(out=(1 << 60, 24, 6)), "BAD_SHAPE")])
def test_delta_scan_refuses_shapes(kw, status):
    d = delta_desc(**kw)
    assert scan(d) == getattr(api, "TAC_ERR_" + status)
    assert scan_backward(d) == getattr(api, "TAC_ERR_" + status)


@pytest.mark.parametrize("name", ["grad_query", "grad_key", "grad_value", "grad_gate", "grad_write"])
def test_delta_scan_backward_refuses_the_gradients_layouts(name):
    assert scan_backward(delta_desc(**{name: (1, 1, 1)})) == api.TAC_ERR_BAD_SHAPE


def test_delta_scan_refuses_addresses():
    assert scan(None) == api.TAC_ERR_NULL and scan_backward(None) == api.TAC_ERR_NULL and step(None) == api.TAC_ERR_NULL
    for i in (0, 1, 2, 3, 4, 7, 11):                                   # inputs, out, workspace
        assert scan(delta_desc(), {i: None}) == api.TAC_ERR_NULL
    for i in (9, 10):                                                  # states and updates come together
        assert scan(delta_desc(), {i: None}) == api.TAC_ERR_NULL
    for i in (0, 1, 2, 3, 4, 7):
        assert scan(delta_desc(), {i: ODD}) == api.TAC_ERR_ALIGN
    for i in (5, 6, 8, 9, 10):
        assert scan(delta_desc(), {i: P + 2}) == api.TAC_ERR_ALIGN
    assert scan(delta_desc(), {11: P + 8}) == api.TAC_ERR_ALIGN
    for i in (0, 1, 2, 3, 4, 6, 7, 8, 10, 11, 12, 13, 14, 16):
        assert scan_backward(delta_desc(), {i: None}) == api.TAC_ERR_NULL, i
    for i in (0, 1, 2, 3, 4, 8, 10, 11, 12, 13, 14):
        assert scan_backward(delta_desc(), {i: ODD}) == api.TAC_ERR_ALIGN, i
    for i in (5, 6, 7, 9, 15):
        assert scan_backward(delta_desc(), {i: P + 2}) == api.TAC_ERR_ALIGN, i
    assert scan_backward(delta_desc(), {16: P + 8}) == api.TAC_ERR_ALIGN


def test_outputs_on_inputs_are_refused():
    apart = {i: P + 4096 * (i + 1) for i in range(17)}
    one = lambda f, desc, n, moved, **kw: f(desc, {**{i: apart[i] for i in range(n)}, **moved}, **kw)
    for i in (0, 1, 2, 3, 4, 6, 8, 9, 10):                             # inputs, h0, and other outputs
        assert one(scan, delta_desc(), 12, {7: apart[i]}) == api.TAC_ERR_BAD_PARAM
    for i in (0, 1, 2, 6, 8, 10):                                      # states
        assert one(scan, delta_desc(), 12, {9: apart[i]}) == api.TAC_ERR_BAD_PARAM
    for w in (10, 11, 12, 13, 14):
        for r in (0, 1, 2, 3, 4, 6, 7, 8, 9, 15):
            assert one(scan_backward, delta_desc(), 17, {w: apart[r]}) == api.TAC_ERR_BAD_PARAM
    assert one(scan_backward, delta_desc(), 17, {10: apart[11]}) == api.TAC_ERR_BAD_PARAM
    a = {i: apart[i] for i in range(9) if i != 6}
    for i in range(6):
        assert step(delta_desc(T=1), {**a, 8: apart[i]}) == api.TAC_ERR_BAD_PARAM


def test_delta_step_refuses():
    one = delta_desc(T=1)
    assert step(delta_desc()) == api.TAC_ERR_BAD_SHAPE                 # more than one step
    for n in (0, -1, 1 << 31):
        assert step(one, n_slots=n) == api.TAC_ERR_BAD_SHAPE
    assert step(one, {7: None}, n_slots=2) == api.TAC_ERR_BAD_SHAPE    # fewer slots than sequences, and none named
    for i in (0, 1, 2, 3, 4, 5, 8):
        assert step(one, {i: None}) == api.TAC_ERR_NULL
    for i in (0, 2, 4, 8):
        assert step(one, {i: ODD}) == api.TAC_ERR_ALIGN
    for i in (5, 7):
        assert step(one, {i: P + 2}) == api.TAC_ERR_ALIGN
    assert step(delta_desc(T=1, value=(0, 5, 6))) == api.TAC_ERR_BAD_SHAPE


def test_workspaces():
    for f in (api.lib().tac_delta_scan_workspace_bytes, api.lib().tac_delta_scan_backward_workspace_bytes):
        assert f(ctypes.byref(delta_desc(T=0))) == 0 and f(None) == 0
        assert f(ctypes.byref(delta_desc(T=64))) > 0 and f(ctypes.byref(delta_desc(T=65))) > f(ctypes.byref(delta_desc(T=64)))
        assert f(ctypes.byref(delta_desc(T=64))) % 16 == 0
