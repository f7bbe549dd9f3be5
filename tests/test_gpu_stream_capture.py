"""Calls on a stream that a capture has forked to (stream=side), replayed between eager calls."""
import pytest
import torch

from paper_2606_01294_amd import ccq
from test_gpu_stream_memory import LATE, NAMES, layer, mixer, tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", [n for n in NAMES if n not in ("delta_step", "conv_step", "decode")])
def test_forked_capture(name):
    """(The step forms move their state on in place: a replay is another step.)"""
    print(name, flush=True)
    f, args = {**layer(), **mixer()}[name]
    ref = {n: t.clone() for n, t in tensors(f(*args)).items()}
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        got = tensors(f(*args, stream=side))
        torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        for t in got.values():
            t.fill_(0)
        junk = [torch.full((1 << 20,), 255, dtype=torch.uint8, device="cuda") for _ in range(8)]
        torch.cuda._sleep(LATE // 20)
        graph.replay()
        again = tensors(f(*args))
        del junk
        torch.cuda.synchronize()
        for n in ref:
            assert torch.equal(got[n], ref[n]) and torch.equal(again[n], ref[n]), n
