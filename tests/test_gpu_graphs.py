"""Calls captured into graphs without a workspace of the caller's: each graph has its own, which
every replay leaves as it needs it, whatever was replayed before or runs beside it."""
import pytest
import torch

from gpu_util import announce, torch_or_skip

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def hd_gpu():
    torch_or_skip()
    import paper_2506_09282_amd as hd
    return hd


def calls(hd):
    """name, inputs to overwrite, the call; each needs a workspace that begins zeroed."""
    g = torch.Generator().manual_seed(1)
    s = torch.randn(3, 30000, generator=g).cuda()
    y = torch.tensor([5, 29999, 17], dtype=torch.int32, device="cuda")
    yield "logprobs", s, lambda: [v for v in hd.logprobs(s, y, top=5)]
    B = torch.randn(561, 10240, generator=g).cuda()
    C = torch.randn(6, 10240, generator=g).sign().cuda()
    X = torch.randn(8, 561, generator=g).cuda()
    assert hd.infer_workspace_bytes(8, 561, 10240, 6, F32) > 0
    yield "infer", X, lambda: list(hd.infer(X, B, C, return_scores=True, deterministic=True))
    model = hd.pack_model(B, C)
    yield "infer_packed", X, lambda: list(hd.infer_packed(X, model, return_scores=True,
                                                          deterministic=True))


def spoil(hd, before):
    """What memory that a capture left to the cache could hold."""
    for key, ws in hd._ws_cache.items():
        if key not in before:
            ws.fill_(255)
    torch.cuda.synchronize()


@pytest.mark.parametrize("which", ["logprobs", "infer", "infer_packed"])
def test_graphs_in_any_order(which):
    hd = hd_gpu()
    name, x, call = next(c for c in calls(hd) if c[0] == which)
    announce(f"graphs of {name}")
    inputs = [torch.randn(x.shape, generator=torch.Generator().manual_seed(k)).cuda()
              for k in range(4)]
    want = []
    for v in inputs:
        x.copy_(v)
        want.append([o.clone() for o in call()])
    torch.cuda.synchronize()
    before = set(hd._ws_cache)
    stream = torch.cuda.Stream()
    graphs, outs = [], []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=stream):
            outs.append(call())
    assert set(hd._ws_cache) == before  # (a capture has not run: it leaves nothing to others)
    spoil(hd, before)
    for k, first in enumerate((1, 0, 0, 1)):  # the second one first
        x.copy_(inputs[k])
        for i in (first, 1 - first):
            graphs[i].replay()
            torch.cuda.synchronize()
            for a, b in zip(outs[i], want[k]):
                assert torch.equal(a, b)
        with torch.cuda.stream(stream):       # eager calls where the capture was
            again = call()
        torch.cuda.synchronize()
        for a, b in zip(again, want[k]):
            assert torch.equal(a, b)


def test_graphs_on_two_streams():
    """Two graphs of one shape, beside each other."""
    hd = hd_gpu()
    _, s, call = next(iter(calls(hd)))
    want = [v.clone() for v in call()]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    graphs, outs = [], []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(call())
    torch.cuda.synchronize()
    for _ in range(20):
        for st, gr in zip(streams, graphs):
            with torch.cuda.stream(st):
                gr.replay()
    torch.cuda.synchronize()
    for out in outs:
        for a, b in zip(out, want):
            assert torch.equal(a, b)
