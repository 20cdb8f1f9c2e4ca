"""GPU tests of graphs that die, as parts of dead cycles of objects, while another graph is captured."""
import gc

import pytest
import torch

from paper_2609_21704_amd import decoder as dec
from paper_2609_21704_amd import rounds
from test_gpu_engine import ragged_prompts
from test_gpu_paged_decoder import config

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Holder:
    """Holds a graph and itself, so only the garbage collector frees it."""

    def __init__(self, graph, freed):
        self.graph, self.me, self.freed = graph, self, freed

    def __del__(self):
        self.freed.append(torch.cuda.is_current_stream_capturing())


@pytest.fixture
def eager_collector():
    old = gc.get_threshold()
    gc.set_threshold(1, 1, 1)
    yield
    gc.set_threshold(*old)
    assert gc.isenabled()


def test_a_graph_that_dies_within_a_capture(eager_collector):
    x, freed = torch.zeros(64, device=DEV), []
    held = [Holder(rounds.captured(lambda: x.add_(1)), freed)]

    def step():
        held.clear()
        for _ in range(100):  # (allocations, at which the collector would run)
            [[] for _ in range(50)]
        x.add_(2)

    g = rounds.captured(step)
    gc.collect()
    assert freed == [False]
    for i in range(3):
        g.replay()
        torch.cuda.synchronize()
        assert bool((x == 2 * (i + 1)).all())


@pytest.mark.parametrize("kind", ["spec", "direct"])
def test_decoders_captured_among_dead_ones(kind, eager_collector):
    cfg = config(2)
    w = dec.DecoderWeights(cfg, DEV)
    prompts = ragged_prompts(cfg, [40, 9], 41)
    make = dec.SpecDecoder if kind == "spec" else dec.DirectDecoder
    outs, held, freed = [], [], []
    for _ in range(3):
        d = make(w, capacity=128, temperature=0.0)
        d.prefill_packed(prompts)
        plain = d.run

        def run():
            if torch.cuda.is_current_stream_capturing():
                held.clear()  # the graph of the decoder before this one
            plain()

        d.run = run
        d.capture()
        for _ in range(3):
            d.replay()
        torch.cuda.synchronize()
        outs.append((d.out_len.tolist(), d.out_tokens[:, :4].tolist()))
        held.append(Holder(d.graph, freed))
        d.graph = None
    held.clear()
    gc.collect()
    assert freed == [False] * 3 and outs[0] == outs[1] == outs[2]


def test_the_collector_is_left_as_it_was():
    x = torch.zeros(8, device=DEV)
    gc.disable()
    try:
        rounds.captured(lambda: x.add_(1))
        assert not gc.isenabled()
    finally:
        gc.enable()
    rounds.captured(lambda: x.add_(1))
    assert gc.isenabled()
