"""The head norm and the gated delta rule on a stream that is not torch's current one, and from two threads at once: results and scratch belong to the stream that is given."""
import threading

import pytest
import torch

import delta_util as O
from paper_2603_13810_amd import api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAMES = ("query", "key", "value", "gate", "write")


def calls(seed=5):
    x, h0 = O.delta_inputs(150, 2, 2, 4, 32, 48, torch.bfloat16, seed)
    args = [x[n] for n in NAMES]
    q, k = args[0].flatten(0, 1), args[1].flatten(0, 1)
    how = dict(eps=1e-6, positions=torch.arange(q.shape[0], dtype=torch.int32, device=DEV))
    kept = api.tac_delta_scan(*args, h0=h0, want_kept=True)
    grad = torch.ones_like(args[2])
    pool = torch.zeros(2, 4, 32, 48, device=DEV)

    def step(s):
        pool.zero_()
        torch.cuda.synchronize()
        return [api.tac_delta_step(*[a[0] for a in args], pool, stream=s)]

    return {
        "heads": lambda s: list(api.tac_head_norm(q, k, **how, stream=s).values()),
        "heads_backward": lambda s: list(api.tac_head_norm_backward(q, k, None, None, q, k, **how, stream=s).values()),
        "scan": lambda s: list(api.tac_delta_scan(*args, h0=h0, want_kept=True, stream=s).values())[:2],
        "scan_backward": lambda s: list(api.tac_delta_scan_backward(*args, kept["states"], kept["updates"], grad, stream=s).values()),
        "step": step,
    }


@pytest.mark.parametrize("name", ["heads", "heads_backward", "scan", "scan_backward", "step"])
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


def test_calls_of_two_threads_at_once():
    sets = [calls(20), calls(21)]
    torch.cuda.synchronize()
    want = [{n: [t.clone() for t in c[n](None)] for n in ("heads", "scan", "scan_backward")} for c in sets]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        stream = torch.cuda.Stream()
        for _ in range(20):
            for n in want[i]:
                got = sets[i][n](stream.cuda_stream)
                stream.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want[i][n])):
                    wrong.append((i, n))
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_two_captured_graphs_side_by_side():
    """Each has scratch of its own."""
    graphs, results, want = [], [], []
    for seed in (30, 31):
        c = calls(seed)
        call = lambda c=c: c["scan"](None) + c["scan_backward"](None)
        want.append([t.clone() for t in call()])
        torch.cuda.synchronize()
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            results.append(call())
        graphs.append((graph, c))
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(5):
        for (graph, _), s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for r, w in zip(results, want):
            assert all(torch.equal(a, b) for a, b in zip(r, w))
            for t in r:
                t.zero_()
        torch.cuda.synchronize()
