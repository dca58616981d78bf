"""The attention layer's own steps around the operators, without a device."""
import pytest
import torch

from paper_2605_10793_amd.layer import AttentionLayer


class Cache:
    heads, device = 2, 0


class Streams:
    """torch.cuda's streams as far as the layer uses them: what waits for what, and when the calibrator reads."""

    def __init__(self, monkeypatch, current):
        self.done = []

        class Stream:
            def __init__(stream, handle, device=None):
                stream.cuda_stream = handle

            def wait_stream(stream, other):
                self.done.append((stream.cuda_stream, "waits for", other.cuda_stream))

        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream(current))
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: current, raising=False)
        monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: Stream(0))
        monkeypatch.setattr(torch.cuda, "ExternalStream", Stream)


class Calibrator:
    device = 0

    def __init__(self, stream, done):
        self.stream, self.done = stream, done

    def step_batch_heads(self, x, head0, heads):
        self.done.append(("reads", x.shape, heads))


def layer_of(calibrator=None, sequences=2):
    layer = AttentionLayer(None, None, None, Cache(), torch.zeros(sequences, 3, dtype=torch.int32), calibrator=calibrator)
    layer._last = None, None, torch.zeros(5, 2, 64), torch.zeros(5, 2, 64), None, torch.zeros(5, 4, 64)
    return layer


@pytest.mark.parametrize("current,of_calibrator", [(0x10, 0x20), (0, 0x20), (0x10, 0)])
def test_the_calibrator_s_stream_waits_and_is_waited_for(monkeypatch, current, of_calibrator):
    """It reads what the current stream writes, in memory that the current stream's allocator may give out again."""
    streams = Streams(monkeypatch, current)
    layer = layer_of(Calibrator(of_calibrator, streams.done))
    layer.commit(torch.tensor([0, 2, 5], dtype=torch.int32))
    assert streams.done == [(of_calibrator, "waits for", current), ("reads", (5, 256), 4), (current, "waits for", of_calibrator)]
    assert layer.prefix.tolist() == [2, 3]


def test_one_stream_waits_for_nothing(monkeypatch):
    streams = Streams(monkeypatch, 0x10)
    layer_of(Calibrator(0x10, streams.done)).commit(torch.tensor([0, 2, 5], dtype=torch.int32))
    assert streams.done == [("reads", (5, 256), 4)]


def test_a_calibrator_of_another_device_is_refused():
    other = Calibrator(0, [])
    other.device = 1
    with pytest.raises(ValueError):
        layer_of(other)


@pytest.mark.parametrize("tokens,sequences,max_query", [(100, 1, 64), (129, 2, 64), (7, 2, 3)])
def test_more_tokens_than_have_results_are_refused(tokens, sequences, max_query):
    """Before any of them is in the cache."""
    with pytest.raises(ValueError):
        layer_of(sequences=sequences).step(torch.zeros(tokens, 8, 64), torch.zeros(sequences + 1, dtype=torch.int32), max_query=max_query)
