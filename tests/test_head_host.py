"""Dense operators, without a GPU: sizes, refusals before anything is launched, the formulas' gradients against differences."""
import ctypes
import os
import re

import numpy as np
import pytest

import head_util as U
from paper_2603_13810_amd import api

HEADER = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "tac.h")).read()
P, ODD = 1 << 20, (1 << 20) + 1              # addresses that are never read: nothing is launched


def call(name, *args):
    return getattr(api.lib(), name)(*args)


@pytest.mark.parametrize("struct", [api.tac_quantize_desc_t, api.tac_norm_desc_t, api.tac_product_desc_t, api.tac_scan_desc_t])
def test_struct_layouts_match_the_header(struct):
    name = struct.__name__
    body = HEADER[HEADER.index("typedef struct %s {" % name[:-2]):HEADER.index("} %s;" % name)]
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    kinds = {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float}
    fields = [(n.strip(), kinds[k]) for k, names in re.findall(r"(int32_t|int64_t|float)\s+([^;]+);", body) for n in names.split(",")]
    assert fields == list(struct._fields_)


def test_constants_match_the_header():
    for n in ("TAC_SCALE_BLOCK", "TAC_SCAN_CHUNK", "TAC_NORM_MAX_COLS"):
        assert int(re.search(r"#define %s (\d+)" % n, HEADER).group(1)) == getattr(api, n)


def test_sizes_of_8bit_matrices():
    assert api.tac_code_bytes(3, 1) == 3 * 128 and api.tac_code_bytes(3, 128) == 3 * 128 and api.tac_code_bytes(3, 129) == 3 * 256
    assert api.tac_scale_bytes(3, 1) == 12 and api.tac_scale_bytes(3, 512) == 12 and api.tac_scale_bytes(3, 513) == 24
    for bad in ((0, 5), (5, 0), (-1, 5)):
        assert api.tac_code_bytes(*bad) == 0 and api.tac_scale_bytes(*bad) == 0


def quantize(src=P, src_scales=P, codes=P, scales=P, codes_t=P, scales_t=P, desc=True, **kw):
    d = dict(rows=5, cols=7, src_stride=7, dtype=api.TAC_BF16, block=0)
    d.update(kw)
    return call("tac_quantize", ctypes.byref(api.tac_quantize_desc_t(**d)) if desc else None, src, src_scales, codes, scales, codes_t,
                scales_t, None)


@pytest.mark.parametrize("kw,status", [
    (dict(desc=False), "NULL"), (dict(src=None), "NULL"), (dict(codes=None), "NULL"), (dict(scales_t=None), "NULL"),
    (dict(codes=None, scales=None, codes_t=None, scales_t=None), "NULL"), (dict(dtype=api.TAC_SCALED, src_scales=None), "NULL"),
    (dict(rows=0), "BAD_SHAPE"), (dict(cols=-1), "BAD_SHAPE"), (dict(src_stride=6), "BAD_SHAPE"), (dict(src_stride=-7), "BAD_SHAPE"),
    (dict(rows=1 << 31), "BAD_SHAPE"), (dict(rows=1 << 30, cols=2048, src_stride=2048), "BAD_SHAPE"), (dict(src_stride=1 << 60), "BAD_SHAPE"),
    (dict(dtype=3), "BAD_PARAM"), (dict(block=2), "BAD_PARAM"),
    (dict(src=ODD), "ALIGN"), (dict(codes=P + 8), "ALIGN"), (dict(scales=P + 2), "ALIGN"), (dict(codes_t=P + 4), "ALIGN"),
    (dict(dtype=api.TAC_SCALED, src=P + 8), "ALIGN"), (dict(dtype=api.TAC_FP32, src=P + 2), "ALIGN")])
def test_quantize_refuses(kw, status):
    assert quantize(**kw) == getattr(api, "TAC_ERR_" + status)


@pytest.mark.parametrize("args,status", [
    ((0, 7, P, P, 0, P, 7), "BAD_SHAPE"), ((5, 7, P, P, 0, P, 6), "BAD_SHAPE"), ((5, 7, None, P, 0, P, 7), "NULL"),
    ((5, 7, P, P, 2, P, 7), "BAD_PARAM"), ((5, 7, P + 4, P, 0, P, 7), "ALIGN"), ((5, 7, P, P, 0, P + 2, 7), "ALIGN")])
def test_dequantize_refuses(args, status):
    assert call("tac_dequantize", *args, None) == getattr(api, "TAC_ERR_" + status)


def norm(desc=True, x=P, residual=P, gain=P, h=P, y=P, codes=P, scales=P, rstd=P, **kw):
    d = dict(rows=5, x_stride=8, residual_stride=8, h_stride=8, y_stride=8, cols=8, dtype=api.TAC_BF16, eps=1e-5)
    d.update(kw)
    return call("tac_residual_norm", ctypes.byref(api.tac_norm_desc_t(**d)) if desc else None, x, residual, gain, h, y, codes, scales,
                rstd, None)


@pytest.mark.parametrize("kw,status", [
    (dict(desc=False), "NULL"), (dict(x=None), "NULL"), (dict(scales=None), "NULL"), (dict(codes=None), "NULL"),
    (dict(h=None, y=None, codes=None, scales=None, rstd=None), "NULL"),
    (dict(rows=0), "BAD_SHAPE"), (dict(cols=0), "BAD_SHAPE"), (dict(x_stride=7), "BAD_SHAPE"), (dict(residual_stride=0), "BAD_SHAPE"),
    (dict(h_stride=7), "BAD_SHAPE"), (dict(y_stride=-8), "BAD_SHAPE"),
    (dict(cols=32769, x_stride=40000, residual_stride=40000, h_stride=40000, y_stride=40000), "UNSUPPORTED"),
    (dict(dtype=2), "BAD_PARAM"), (dict(eps=0.0), "BAD_PARAM"), (dict(eps=float("nan")), "BAD_PARAM"), (dict(eps=float("inf")), "BAD_PARAM"),
    (dict(x=ODD), "ALIGN"), (dict(gain=P + 2), "ALIGN"), (dict(codes=P + 8), "ALIGN"), (dict(rstd=P + 1), "ALIGN")])
def test_norm_refuses(kw, status):
    assert norm(**kw) == getattr(api, "TAC_ERR_" + status)


def norm_backward(desc=True, h=P, gain=P, rstd=P, grad_y=P, grad_h=P, grad_x=P, grad_gain=P, workspace=P, **kw):
    d = dict(rows=5, x_stride=8, residual_stride=8, h_stride=8, y_stride=8, cols=8, dtype=api.TAC_BF16, eps=1e-5)
    d.update(kw)
    return call("tac_residual_norm_backward", ctypes.byref(api.tac_norm_desc_t(**d)) if desc else None, h, gain, rstd, grad_y, grad_h,
                grad_x, grad_gain, workspace, None)


@pytest.mark.parametrize("kw,status", [
    (dict(desc=False), "NULL"), (dict(h=None), "NULL"), (dict(rstd=None), "NULL"), (dict(grad_y=None), "NULL"), (dict(grad_x=None), "NULL"),
    (dict(workspace=None), "NULL"), (dict(cols=0), "BAD_SHAPE"), (dict(x_stride=7), "BAD_SHAPE"), (dict(y_stride=3), "BAD_SHAPE"),
    (dict(grad_h=ODD), "ALIGN"), (dict(grad_gain=P + 2), "ALIGN"), (dict(workspace=P + 4), "ALIGN")])
def test_norm_backward_refuses(kw, status):
    assert norm_backward(**kw) == getattr(api, "TAC_ERR_" + status)


def product(desc=True, a=P, a_scales=P, b=P, b_scales=P, bias=P, y=P, workspace=P, **kw):
    d = dict(M=4, N=6, K=9, y_stride=6, dtype=api.TAC_BF16)
    d.update(kw)
    return call("tac_scaled_product", ctypes.byref(api.tac_product_desc_t(**d)) if desc else None, a, a_scales, b, b_scales, bias, y,
                workspace, None)


@pytest.mark.parametrize("kw,status", [
    (dict(desc=False), "NULL"), (dict(a=None), "NULL"), (dict(a_scales=None), "NULL"), (dict(b=None), "NULL"), (dict(y=None), "NULL"),
    (dict(M=0), "BAD_SHAPE"), (dict(N=0), "BAD_SHAPE"), (dict(K=0), "BAD_SHAPE"), (dict(K=1 << 31), "BAD_SHAPE"), (dict(y_stride=5), "BAD_SHAPE"),
    (dict(dtype=2), "BAD_PARAM"), (dict(a=P + 8), "ALIGN"), (dict(b_scales=P + 1), "ALIGN"), (dict(bias=P + 2), "ALIGN"), (dict(y=ODD), "ALIGN"),
    (dict(workspace=P + 8), "ALIGN")])
def test_product_refuses(kw, status):
    assert product(**kw) == getattr(api, "TAC_ERR_" + status)


SCAN = dict(T=6, B=2, D=8, in_stride_t=16, in_stride_b=8, out_stride_t=16, out_stride_b=8, grad_stride_t=16, grad_stride_b=8,
            dtype=api.TAC_BF16)


def scan(desc=True, gate=P, value=P, lengths=P, h0=P, out=P, h_last=P, states=P, workspace=P, **kw):
    d = api.tac_scan_desc_t(**dict(SCAN, **kw))
    return call("tac_gated_scan", ctypes.byref(d) if desc else None, gate, value, lengths, h0, out, h_last, states, workspace, None)


def scan_backward(desc=True, gate=P, value=P, lengths=P, states=P, grad_out=P, grad_h_last=P, grad_gate=P, grad_value=P, grad_h0=P,
                  workspace=P, **kw):
    d = api.tac_scan_desc_t(**dict(SCAN, **kw))
    return call("tac_gated_scan_backward", ctypes.byref(d) if desc else None, gate, value, lengths, states, grad_out, grad_h_last,
                grad_gate, grad_value, grad_h0, workspace, None)


SCAN_REFUSALS = [
    (dict(desc=False), "NULL"), (dict(gate=None), "NULL"), (dict(value=None), "NULL"),
    (dict(T=0), "BAD_SHAPE"), (dict(B=0), "BAD_SHAPE"), (dict(B=65536), "BAD_SHAPE"), (dict(D=-4), "BAD_SHAPE"), (dict(in_stride_t=7), "BAD_SHAPE"),
    (dict(in_stride_b=7), "BAD_SHAPE"), (dict(out_stride_t=0), "BAD_SHAPE"), (dict(out_stride_b=-8), "BAD_SHAPE"), (dict(dtype=2), "BAD_PARAM"),
    (dict(gate=ODD), "ALIGN"), (dict(lengths=P + 2), "ALIGN"), (dict(states=P + 1), "ALIGN"), (dict(workspace=P + 8), "ALIGN")]


@pytest.mark.parametrize("kw,status", SCAN_REFUSALS + [(dict(out=None), "NULL"), (dict(h_last=P + 2), "ALIGN")])
def test_scan_refuses(kw, status):
    assert scan(**kw) == getattr(api, "TAC_ERR_" + status)


@pytest.mark.parametrize("kw,status", SCAN_REFUSALS + [
    (dict(states=None), "NULL"), (dict(grad_out=None), "NULL"), (dict(grad_gate=None), "NULL"), (dict(grad_value=None), "NULL"),
    (dict(grad_stride_t=7), "BAD_SHAPE"), (dict(grad_stride_b=0), "BAD_SHAPE"), (dict(grad_value=ODD), "ALIGN"), (dict(grad_h0=P + 2), "ALIGN")])
def test_scan_backward_refuses(kw, status):
    assert scan_backward(**kw) == getattr(api, "TAC_ERR_" + status)


def step(desc=True, gate=P, value=P, pool=P, n_slots=9, slots=P, out=P, **kw):
    d = api.tac_scan_desc_t(**dict(SCAN, T=1, **kw)) if "T" not in kw else api.tac_scan_desc_t(**dict(SCAN, **kw))
    return call("tac_gated_step", ctypes.byref(d) if desc else None, gate, value, pool, n_slots, slots, out, None)


@pytest.mark.parametrize("kw,status", [
    (dict(desc=False), "NULL"), (dict(pool=None), "NULL"), (dict(out=None), "NULL"), (dict(T=2), "BAD_SHAPE"), (dict(n_slots=0), "BAD_SHAPE"),
    (dict(slots=None, n_slots=1), "BAD_SHAPE"), (dict(in_stride_b=4), "BAD_SHAPE"), (dict(pool=P + 2), "ALIGN"), (dict(slots=P + 1), "ALIGN")])
def test_step_refuses(kw, status):
    assert step(**kw) == getattr(api, "TAC_ERR_" + status)


def test_binding_refuses_what_the_library_cannot_see():
    import torch
    m = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        api.tac_quantize(m)                                     # not a device tensor
    with pytest.raises(ValueError):
        api.tac_residual_norm(m, eps=1e-5)
    with pytest.raises(ValueError):
        api.tac_residual_norm(m[0], eps=1e-5)
    with pytest.raises(ValueError):
        api.tac_gated_scan(m, m)
    with pytest.raises(ValueError):
        api.tac_gated_step(m, m, m[0])
    with pytest.raises(ValueError):
        api.tac_scaled_product(m.to(torch.uint8), m.to(torch.uint8), m.to(torch.uint8), m.to(torch.uint8), 8)


def differences(f, x, eps=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        keep = x[i]
        x[i] = keep + eps
        up = f()
        x[i] = keep - eps
        g[i] = (up - f()) / (2 * eps)
        x[i] = keep
    return g


def test_norm_formulas_gradient_against_differences():
    r = np.random.default_rng(1)
    x, res, gain, gy, gh = (r.standard_normal(s) for s in ((3, 7), (3, 7), (7,), (3, 7), (3, 7)))

    def loss():
        s, _, y = U.norm(x, res, gain, 1e-3)
        return (y * gy).sum() + (s * gh).sum()
    s, rstd, _ = U.norm(x, res, gain, 1e-3)
    gx, gg = U.norm_backward(s, rstd, gain, gy, gh)
    # central differences: error eps^2 |f'''| / 6 + rounding 2^-52 |f| / eps, both below 1e-8 here
    assert np.abs(differences(loss, x) - gx).max() < 1e-7
    assert np.abs(differences(loss, res) - gx).max() < 1e-7
    assert np.abs(differences(loss, gain) - gg).max() < 1e-7


@pytest.mark.parametrize("lengths", [None, (5, 0, 3)])
def test_scan_formulas_gradient_against_differences(lengths):
    r = np.random.default_rng(2)
    g, u, go = (r.standard_normal((5, 3, 4)) for _ in range(3))
    h0, gl = r.standard_normal((3, 4)), r.standard_normal((3, 4))
    n = None if lengths is None else np.array(lengths)

    def loss():
        out, _, last = U.scan(g, u, n, h0)
        return (out * go).sum() + (last * gl).sum()
    _, before, _ = U.scan(g, u, n, h0)
    gg, gv, g0 = U.scan_backward(g, u, before, go, n, gl)
    assert np.abs(differences(loss, g) - gg).max() < 1e-7
    assert np.abs(differences(loss, u) - gv).max() < 1e-7
    assert np.abs(differences(loss, h0) - g0).max() < 1e-7


def test_8bit_oracle_is_the_nearest_number():
    # all 127 magnitudes of e4m3, and every midpoint between neighbours goes to the even code
    codes = np.arange(127)
    x, f = codes >> 3, (codes & 7).astype(float)
    all_values = np.where(x == 0, f * 2.0 ** -9, (8 + f) * np.exp2(x - 10.0))
    assert np.array_equal(U.e4m3(all_values), all_values) and all_values[-1] == 448
    mid = (all_values[1:] + all_values[:-1]) / 2
    assert np.array_equal(U.e4m3(mid), np.where(codes[1:] % 2 == 0, all_values[1:], all_values[:-1]))
    v = np.array([[448.0, 1.0], [449.0, 1.0], [0.0, 0.0], [2.0 ** -140, 0.0]])
    assert U.block_exponents(v)[:, 0].tolist() == [0, 1, -127, -127]


def test_laying_8bit_values_out_again_is_exact_above_the_subnormals():
    r = np.random.default_rng(3)
    v, _ = U.quantized(r.standard_normal((128, 256)))
    again, e = U.quantized(np.ascontiguousarray(v.T))
    unit = np.exp2(np.repeat(e, 128, axis=1).astype(float))[:, :128]
    normal = np.abs(v.T) >= 2.0 ** -6 * unit
    assert normal.mean() > 0.97 and np.array_equal(again[normal], v.T[normal])
    assert (np.abs(again - v.T) <= 2.0 ** -10 * unit).all()


CALLS = {
    "quantize": lambda t, s: api.tac_quantize(t, stream=s),
    "quantize codes": lambda t, s: api.tac_quantize((t, t), cols=8, stream=s),
    "dequantize": lambda t, s: api.tac_dequantize((t, t), 8, stream=s),
    "residual_norm": lambda t, s: api.tac_residual_norm(t, eps=1e-5, stream=s),
    "residual_norm_backward": lambda t, s: api.tac_residual_norm_backward(t, None, t, t, stream=s),
    "scaled_product": lambda t, s: api.tac_scaled_product(t, t, t, t, 8, stream=s),
    "gated_scan": lambda t, s: api.tac_gated_scan(t, t, stream=s),
    "gated_scan_backward": lambda t, s: api.tac_gated_scan_backward(t, t, t, t, stream=s),
    "gated_step": lambda t, s: api.tac_gated_step(t, t, t, stream=s),
}


@pytest.mark.parametrize("name", CALLS)
def test_a_given_stream_is_one_of_the_tensors_device(name, monkeypatch):
    import contextlib
    import types
    import torch
    seen, inside = [], []

    class Native:
        def __getattr__(self, function):
            return lambda *args: (function, list(inside))

    @contextlib.contextmanager
    def current(stream):
        inside.append(stream)
        yield
        inside.pop()
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: seen.append((handle, device)) or (handle, device))
    monkeypatch.setattr(torch.cuda, "stream", current)
    monkeypatch.setattr(api, "_native", Native)
    tensor = types.SimpleNamespace(device=torch.device("cuda:1"))        # not the current device
    function, streams = CALLS[name](tensor, 77)
    assert function == name.split()[0] and streams == seen == [(77, torch.device("cuda:1"))]
    function, streams = CALLS[name](tensor, None)
    assert function == name.split()[0] and streams == [] and len(seen) == 1


@pytest.mark.parametrize("name", CALLS)
def test_a_stream_does_not_change_what_is_refused(name):
    import torch
    with pytest.raises(ValueError):
        CALLS[name](torch.zeros(4, 8), 77)
    with pytest.raises((ValueError, TypeError)):
        CALLS[name](None, 77)


@pytest.mark.parametrize("torch_is", ["missing", "without headers"])
def test_the_library_is_built_without_torchs_headers(torch_is, tmp_path, monkeypatch):
    import subprocess
    import sys
    import types
    from paper_2603_13810_amd import build
    stale, ran = tmp_path / "_operators.so", []
    stale.write_text("of an earlier library")
    monkeypatch.setattr(build, "OPERATORS", str(stale))
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libtac.so"))
    monkeypatch.setattr(build, "SOURCES", ["tac_head_api.hip"])
    monkeypatch.setattr(build, "CSRC", str(tmp_path))
    (tmp_path / "tac_head_api.hip").write_text("")

    def link(cmd):
        ran.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()
    monkeypatch.setattr(subprocess, "run", lambda cmd, **kw: types.SimpleNamespace(stdout="", returncode=0))
    monkeypatch.setattr(subprocess, "check_call", link)
    fake = types.ModuleType("torch")
    fake.__file__ = str(tmp_path / "torch" / "__init__.py")
    monkeypatch.setitem(sys.modules, "torch", None if torch_is == "missing" else fake)
    assert build.build(verbose=False) == str(tmp_path / "libtac.so") and os.path.exists(build.LIB)
    assert len(ran) == 1 and not stale.exists()
