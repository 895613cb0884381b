"""Calls on a stream that a capture has forked to, with memory of their own: the
graph's replays, other work in between, give what the calls give."""
import pytest
import torch

import synth
import test_gpu_foreign_streams as eight
from _gpu_util import Dev
from paper_2609_35587_amd import hwsel

pytestmark = pytest.mark.gpu
data = eight.data


def replayed(call):
    want = [t.clone() for t in call(None)]
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        got = call(side)
        main.wait_stream(side)
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert all(torch.equal(a, b) for a, b in zip(call(None), want))


@pytest.mark.parametrize("name", eight.CALLS)
def test_forked_in_a_capture(name, data):
    replayed(lambda s: eight.tensors(eight.CALLS[name](data, s)))


def test_scoring_forked_in_a_capture():
    w = synth.workload("tiny")
    d = Dev(w)
    X, packed = d.features(64), hwsel.hwsel_forest_pack(d.forest)
    replayed(lambda s: [hwsel.hwsel_forest_score(d.forest, X, packed=packed, stream=s)])
