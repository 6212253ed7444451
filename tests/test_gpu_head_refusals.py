"""What the dense operators' Python calls refuse before anything is launched: types, shapes, strides, what is no tensor, what the library refuses."""
import pytest
import torch

from paper_2603_13810_amd import api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def f32(*shape):
    return torch.zeros(shape, device=DEV)


def u8(*shape):
    return torch.zeros(shape, device=DEV, dtype=torch.uint8)


def matrix(rows, cols):
    return u8(rows, -(-cols // 128) * 128), u8(rows, -(-cols // 512) * 4)


VALUE = [
    lambda: api.tac_quantize(f32(4, 8).half()),
    lambda: api.tac_quantize(f32(4, 8).t()),
    lambda: api.tac_quantize(f32(4)),
    lambda: api.tac_quantize(f32(4, 8).cpu()),
    lambda: api.tac_quantize(matrix(4, 8)),
    lambda: api.tac_quantize((u8(4, 127), u8(4, 4)), cols=8),
    lambda: api.tac_quantize((u8(4, 128), None), cols=0),
    lambda: api.tac_quantize([[1.0]]),
    lambda: api.tac_dequantize(matrix(4, 8), 200),
    lambda: api.tac_dequantize(matrix(4, 8), -1),
    lambda: api.tac_dequantize(matrix(4, 8), 8, dtype=torch.float16),
    lambda: api.tac_dequantize(matrix(4, 8), 8, dtype="float32"),
    lambda: api.tac_dequantize(matrix(4, 8), 8, out=f32(4, 9)),
    lambda: api.tac_residual_norm(f32(4, 8), f32(4, 9), eps=1e-5),
    lambda: api.tac_residual_norm(f32(4, 8), f32(4, 8).bfloat16(), eps=1e-5),
    lambda: api.tac_residual_norm(f32(4, 8), None, f32(8).bfloat16(), eps=1e-5),
    lambda: api.tac_residual_norm(f32(4, 8), None, f32(16)[::2], eps=1e-5),
    lambda: api.tac_residual_norm(f32(4, 8), None, f32(8).cpu(), eps=1e-5),
    lambda: api.tac_residual_norm(None, eps=1e-5),
    lambda: api.tac_residual_norm(f32(4, 8), eps=1e-5, y=f32(8, 4).t()),
    lambda: api.tac_residual_norm_backward(f32(4, 8), None, f32(5), f32(4, 8)),
    lambda: api.tac_residual_norm_backward(f32(4, 8), None, None, f32(4, 8)),
    lambda: api.tac_residual_norm_backward(f32(4, 8), None, f32(4), f32(4, 8), grad_x=f32(4, 7)),
    lambda: api.tac_scaled_product(*matrix(4, 8), *matrix(4, 200), 8),
    lambda: api.tac_scaled_product(*matrix(4, 8), *matrix(4, 8), 0),
    lambda: api.tac_scaled_product(*matrix(4, 8), *matrix(4, 8), 8, bias=f32(5)),
    lambda: api.tac_scaled_product(*matrix(4, 8), *matrix(4, 8), 8, out=f32(4, 5)),
    lambda: api.tac_scaled_product(*matrix(4, 8), *matrix(4, 8), 8, dtype=torch.int32),
    lambda: api.tac_gated_scan(f32(3, 2, 4), f32(3, 2, 5)),
    lambda: api.tac_gated_scan(f32(3, 2, 4), f32(3, 2, 8)[..., :4]),
    lambda: api.tac_gated_scan(f32(3, 2, 4), f32(3, 2, 4), lengths=torch.zeros(2, device=DEV, dtype=torch.int64)),
    lambda: api.tac_gated_scan(f32(3, 2, 4), f32(3, 2, 4), h0=f32(2, 5)),
    lambda: api.tac_gated_scan_backward(f32(3, 2, 4), f32(3, 2, 4), f32(2, 2, 4), f32(3, 2, 4)),
    lambda: api.tac_gated_scan_backward(f32(3, 2, 4), f32(3, 2, 4), f32(1, 2, 4), f32(3, 2, 4), grad_gate=f32(3, 2, 8)[..., :4], grad_value=f32(3, 2, 4)),
    lambda: api.tac_gated_step(f32(2, 4), f32(2, 4), f32(3, 5)),
    lambda: api.tac_gated_step(f32(2, 4), f32(2, 4), f32(3, 4), f32(2)),
    lambda: api.tac_gated_step(f32(2, 4), f32(2, 8)[:, :4], f32(3, 4)),
    lambda: api.tac_gated_step(f32(2, 4), f32(2, 4), f32(3, 4), out=f32(3, 4)),
]


@pytest.mark.parametrize("case", range(len(VALUE)))
def test_values_that_the_binding_refuses(case):
    with pytest.raises(ValueError):
        VALUE[case]()


STATUS = [
    (lambda: api.tac_quantize(f32(4, 8), rows=False), "NULL"),
    (lambda: api.tac_quantize(f32(0, 8)), None),
    (lambda: api.tac_residual_norm(f32(4, 8), eps=0.0), "BAD_PARAM"),
    (lambda: api.tac_residual_norm(f32(4, 8), eps=1e-5, want_y=False), "NULL"),
    (lambda: api.tac_residual_norm(f32(1, 32769), eps=1e-5), "UNSUPPORTED"),
    (lambda: api.tac_residual_norm(f32(4, 8).expand(4, 8)[:1].expand(4, 8), eps=1e-5), "BAD_SHAPE"),
    (lambda: api.tac_gated_scan(f32(0, 2, 4), f32(0, 2, 4)), None),
    (lambda: api.tac_gated_step(f32(4, 4), f32(4, 4), f32(3, 4)), "BAD_SHAPE"),
    (lambda: api.tac_scaled_product(u8(4 * 128 + 1)[1:].view(4, 128), u8(4, 4), *matrix(4, 8), 8), "ALIGN"),
]


@pytest.mark.parametrize("case", range(len(STATUS)))
def test_statuses_of_the_library_become_errors(case):
    call, status = STATUS[case]
    with pytest.raises(api.TacError) as e:
        call()
    if status:
        assert e.value.status == getattr(api, "TAC_ERR_" + status)


def test_outputs_that_are_given_come_back():
    x, h, y = f32(4, 8), f32(4, 8), f32(4, 8)
    r = api.tac_residual_norm(x, x, None, eps=1e-5, h=h, y=y)
    assert r["h"] is h and r["y"] is y and r["scaled"] is None and r["rstd"] is None
    out = f32(3, 2, 4)
    assert api.tac_gated_scan(out, out, out=out)["out"] is out
    g = api.tac_gated_scan_backward(f32(3, 2, 4), f32(3, 2, 4), f32(1, 2, 4), f32(3, 2, 4), grad_gate=f32(3, 2, 8)[..., :4])
    assert g["grad_value"].stride() == g["grad_gate"].stride() == (16, 8, 1)


GIVEN = {
    "dequantize out": lambda t: api.tac_dequantize(matrix(4, 8), 8, out=t),
    "norm h": lambda t: api.tac_residual_norm(f32(4, 8), f32(4, 8), eps=1e-5, h=t),
    "norm y": lambda t: api.tac_residual_norm(f32(4, 8), eps=1e-5, y=t),
    "norm backward grad_x": lambda t: api.tac_residual_norm_backward(f32(4, 8), None, f32(4), f32(4, 8), grad_x=t),
    "product out": lambda t: api.tac_scaled_product(*matrix(4, 8), *matrix(8, 8), 8, out=t),
    "scan out": lambda t: api.tac_gated_scan(f32(2, 2, 8), f32(2, 2, 8), out=t.view(2, 2, 8)),
    "scan backward grad_gate": lambda t: api.tac_gated_scan_backward(f32(2, 2, 8), f32(2, 2, 8), f32(1, 2, 8), f32(2, 2, 8), grad_gate=t.view(2, 2, 8)),
    "scan backward grad_value": lambda t: api.tac_gated_scan_backward(f32(2, 2, 8), f32(2, 2, 8), f32(1, 2, 8), f32(2, 2, 8), grad_value=t.view(2, 2, 8)),
    "step pool": lambda t: api.tac_gated_step(f32(4, 8), f32(4, 8), t),
    "step out": lambda t: api.tac_gated_step(f32(4, 8), f32(4, 8), f32(4, 8), out=t),
}


@pytest.mark.parametrize("name", GIVEN)
def test_a_written_tensor_counts_as_changed_in_place(name):
    t, w = f32(4, 8), f32(4, 8).requires_grad_()
    loss = (w * t).sum()                                     # autograd keeps t
    GIVEN[name](t)
    assert t._version == 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    with torch.inference_mode():
        plain = f32(4, 8)
        GIVEN[name](plain)
    GIVEN[name](plain)                                       # and outside, where torch's own in-place operations refuse it


def test_results_are_not_recorded_by_autograd():
    x = torch.randn(4, 8, device=DEV).requires_grad_()
    got = api.tac_residual_norm(x, x, eps=1e-5, want_rstd=True)
    assert x._version == 0 and not any(got[k].requires_grad for k in ("h", "y", "rstd"))
    before = x.detach().clone()
    api.tac_residual_norm(x, eps=1e-5)
    assert x._version == 0 and torch.equal(x, before)
