"""The dense operators on a stream that is not torch's current one: what a call allocates belongs to the stream that it is given."""
import pytest
import torch

from paper_2603_13810_amd import api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def calls():
    g = torch.Generator(device=DEV).manual_seed(5)
    x = torch.randn(300, 640, generator=g, device=DEV).to(torch.bfloat16)
    w = api.tac_quantize(torch.randn(256, 640, generator=g, device=DEV), tiles=True)["rows"]
    q = api.tac_quantize(x)["rows"]
    seq = torch.randn(400, 2, 128, generator=g, device=DEV)
    norm = api.tac_residual_norm(x, x, None, eps=1e-5, want_rstd=True)
    scan = api.tac_gated_scan(seq, seq, want_states=True)
    pool = torch.zeros(2, 128, device=DEV)

    def step(s):
        pool.zero_()
        torch.cuda.synchronize()
        return [api.tac_gated_step(seq[0], seq[0], pool, stream=s)]

    return {
        "quantize": lambda s: list(api.tac_quantize(x, columns=True, stream=s)["columns"]),
        "dequantize": lambda s: [api.tac_dequantize(q, 640, stream=s)],
        "norm": lambda s: [api.tac_residual_norm(x, x, None, eps=1e-5, stream=s)[k] for k in ("h", "y")],
        "norm_backward": lambda s: list(api.tac_residual_norm_backward(norm["h"], None, norm["rstd"], x, stream=s).values()),
        "product": lambda s: [api.tac_scaled_product(*q, *w, 640, stream=s)],
        "scan": lambda s: [api.tac_gated_scan(seq, seq, stream=s)[k] for k in ("out", "h_last")],
        "scan_backward": lambda s: list(api.tac_gated_scan_backward(seq, seq, scan["states"], seq, stream=s).values()),
        "step": step,
    }


@pytest.mark.parametrize("name", ["quantize", "dequantize", "norm", "norm_backward", "product", "scan", "scan_backward", "step"])
def test_results_of_a_stream_belong_to_it(name):
    call = calls()[name]
    want = call(None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = call(side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    at, size, dtype = [t.data_ptr() for t in got], [t.shape for t in got], [t.dtype for t in got]
    del got
    # the blocks are that stream's: the current one does not get them while work on the other might still read them
    here = [torch.empty(n, dtype=d, device=DEV).data_ptr() for n, d in zip(size, dtype)]
    assert not set(here) & set(at)
    zero = call(0)                              # the default stream by its handle
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(zero, want))
