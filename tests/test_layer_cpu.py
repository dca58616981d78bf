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


@pytest.fixture
def positions_of(monkeypatch):
    """The positions that a step hands to the norms."""
    from paper_2605_10793_amd import layer as module
    seen = []
    monkeypatch.setattr(module.attention, "qk_norm_rotary", lambda plan, q, k, qw, kw, positions, eps: seen.append(positions) or (q, k))
    monkeypatch.setattr(module.attention, "append", lambda *a: None)
    monkeypatch.setattr(module.attention, "tree_attention", lambda q, *a, **more: q)

    def step(prefix, start, tokens, depth=None):
        layer = layer_of(sequences=len(prefix))
        layer.prefix = torch.tensor(prefix, dtype=torch.int32)
        out = layer.step(torch.zeros(tokens, 8, 64), torch.tensor(start, dtype=torch.int32), depth)
        assert out.shape == (tokens, 4, 64) and seen[-1].dtype == torch.int64 and seen[-1].shape == (tokens,)
        layer.commit(torch.tensor(start, dtype=torch.int32))
        return seen[-1].tolist(), layer.prefix.tolist()
    return step


def test_positions_of_a_chain_and_of_a_tree(positions_of):
    assert positions_of([10, 20, 30, 40], [0, 0, 3, 3, 5], 5) == ([20, 21, 22, 40, 41], [10, 23, 30, 42])
    assert positions_of([10, 20], [0, 3, 5], 5, torch.tensor([0, 1, 1, 0, 1])) == ([10, 11, 11, 20, 21], [13, 22])
    assert positions_of([1 << 30, 5], [0, 0, 0], 0) == ([], [1 << 30, 5])


def test_starts_that_do_not_fit_the_tokens(positions_of):
    """Rows of no sequence, entries beyond the rows, negative counts: positions for the rows there are, and counts as the operators take them.
    (What a count repeats must not be written past the rows that there are.)"""
    got, prefix = positions_of([10, 20], [0, 2, 3], 6)
    assert got[:3] == [10, 11, 20] and prefix == [12, 21]
    got, prefix = positions_of([10, 20], [0, 2, 1000], 6)
    assert got == [10, 11, 20, 21, 22, 23] and prefix == [12, 24]
    got, prefix = positions_of([10, 20, 30], [0, 4, 2, 6], 6)
    assert len(got) == 6 and prefix == [14, 20, 34]
    got, prefix = positions_of([10, 20], [-5, -2, 6], 6)
    assert prefix == [10, 26]
