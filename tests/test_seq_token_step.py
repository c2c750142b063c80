"""CPU checks of the recorded step: which stream it is recorded on, and which tokens it takes.  The device, its streams and the graph are stand-ins that keep books."""
import contextlib

import pytest
import torch
from torch.autograd import forward_ad

from paper_2007_06000_amd.binding import XlError
from paper_2007_06000_amd.scan_block import TokenStep

DEVICE = torch.device("meta")           # stands for a GPU that is not the current one


class Stream:
    def __init__(self, device="the current device"):
        self.device = device

    def wait_stream(self, other):
        pass


class Block:
    """What a step needs of a scan block; notes the stream that is current on its device whenever it is called."""
    dev, dtype, width = DEVICE, torch.float32, 8

    def __init__(self, streams):
        self.streams, self.calls = streams, []

    def cache(self, rows):
        return torch.zeros(rows, 3, 16, device=DEVICE), torch.zeros(rows, 16, 4, device=DEVICE)

    def __call__(self, x, state, slots):
        self.calls.append(self.streams[-1])
        return x.clone(), state


@pytest.fixture
def streams(monkeypatch):
    """The stack of current streams, with the calls of torch.cuda that a step makes replaced."""
    stack, recordings = [Stream()], []

    @contextlib.contextmanager
    def use(stream):
        stack.append(stream)
        yield
        stack.pop()

    @contextlib.contextmanager
    def graph(graph, pool=None, stream=None, **more):
        stream = stream or Stream()     # a stream of whichever device is the current one
        recordings.append(stream)
        with use(stream):
            yield

    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "stream", use)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream(device))
    monkeypatch.setattr(torch.cuda, "CUDAGraph", object)
    monkeypatch.setattr(torch.cuda, "graph", graph)
    return stack, recordings


def test_a_step_is_recorded_on_a_stream_of_its_blocks_device(streams):
    stack, recordings = streams
    block = Block(stack)
    TokenStep(block, 2)
    assert len(recordings) == 1 and recordings[0].device == DEVICE
    assert len(block.calls) == 2 and all(s.device == DEVICE for s in block.calls) and block.calls[1] is recordings[0]


class Graph:
    replays = 0

    def replay(self):
        Graph.replays += 1


@pytest.mark.parametrize("shape", [(1, 1, 8), (1, 8), (8,), (2, 2, 8), (2, 1, 1), (3, 1, 8), (2, 8)])
def test_a_step_takes_one_token_for_each_row_and_nothing_else(streams, monkeypatch, shape):
    monkeypatch.setattr(torch.cuda, "CUDAGraph", Graph)
    step = TokenStep(Block(streams[0]), 2)
    before = Graph.replays
    with pytest.raises(XlError):
        step(torch.zeros(shape, device=DEVICE))
    assert Graph.replays == before
    step(torch.zeros(2, 1, 8, device=DEVICE))
    assert Graph.replays == before + 1


def test_a_step_refuses_tokens_that_ask_for_a_gradient(streams, monkeypatch):
    monkeypatch.setattr(torch.cuda, "CUDAGraph", Graph)
    step = TokenStep(Block(streams[0]), 2)
    x = torch.zeros(2, 1, 8, device=DEVICE, requires_grad=True)
    with pytest.raises(XlError):
        step(x)
    with torch.no_grad():
        step(x)
    with forward_ad.dual_level(), pytest.raises(XlError):
        step(forward_ad.make_dual(x.detach(), torch.ones_like(x)))
    assert not step.x.requires_grad
