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


def test_positions_where_starts_fall(positions_of):
    """Starts padded by zeros, sequences of none among others."""
    assert positions_of([10, 20, 30, 40], [0, 1, 3, 0, 0], 3) == ([10, 20, 21], [11, 22, 30, 40])
    assert positions_of([10, 20, 30, 40, 50], [2, 4, 4, 0, 0, 0], 4)[0][2:] == [10, 11]
    assert positions_of([10, 20], [0, 3, 0], 3, torch.tensor([0, 1, 1])) == ([10, 11, 11], [13, 20])
    assert positions_of([10], [0, 3], 3) == ([10, 11, 12], [13])


@pytest.mark.parametrize("sequences", [64, 2000])
def test_positions_of_many_sequences(positions_of, sequences):
    counts = [b % 3 for b in range(sequences)]
    start = [sum(counts[:b]) for b in range(sequences + 1)]
    got, prefix = positions_of([7 * b for b in range(sequences)], start, start[-1])
    assert got == [7 * b + i for b in range(sequences) for i in range(counts[b])] and prefix == [7 * b + n for b, n in enumerate(counts)]


def test_positions_behind_dropped_tokens(monkeypatch, positions_of):
    """The next tokens stand where they would have, through commits and branches, or where those that are left end."""
    from paper_2605_10793_amd import layer as module
    moved, positions = [], []
    monkeypatch.setattr(module.attention, "gather", lambda *a: moved.append(a))
    monkeypatch.setattr(module.attention, "qk_norm_rotary", lambda plan, q, k, qw, kw, p, eps: positions.append(p.tolist()) or (q, k))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    layer = layer_of(sequences=3)
    layer.cache.page_tokens = 16
    layer.prefix = i32([100, 40, 7])
    fused, start = torch.zeros(5, 8, 64), i32([0, 2, 3, 5])
    kept, edges, to = i32(list(range(0, 100, 2)) + list(range(40)) + [6]), i32([0, 50, 90, 91]), torch.ones(3, 3, dtype=torch.int32)
    layer.keep(kept, edges, to, position=layer.position)
    assert moved[0][1:] == (kept, edges, moved[0][3], to) and layer.table is to
    assert layer.prefix.tolist() == [50, 40, 1] and layer.position.tolist() == [100, 40, 7]
    layer.step(fused, start)
    layer.commit(start)
    assert layer.prefix.tolist() == [52, 41, 3] and layer.position.tolist() == [102, 41, 9]
    layer.step(fused, start, depth=torch.tensor([0, 1, 0, 0, 1]))
    layer.branch(torch.tensor([2, 0, 0]), to)
    assert layer.prefix.tolist() == [3, 52, 52] and layer.position.tolist() == [9, 102, 102]
    layer.step(fused, start)
    assert positions == [[100, 101, 40, 7, 8], [102, 103, 41, 9, 10], [9, 10, 102, 102, 103]]
    layer.keep(i32([0, 1, 2]), i32([0, 2, 3, 9]), to)          # (a start behind the tokens that are named)
    assert layer.prefix.tolist() == layer.position.tolist() == [2, 1, 0]
    layer.step(fused, start)
    assert positions[-1] == [2, 3, 1, 0, 1]


@pytest.mark.parametrize("shape", [(3, 2), (3, 4), (2, 3)])
def test_a_branch_into_another_number_of_pages_is_refused(monkeypatch, shape):
    """Before anything is moved."""
    from paper_2605_10793_amd import layer as module
    moved = []
    monkeypatch.setattr(module.attention, "gather", lambda *a: moved.append(a))
    layer = layer_of(sequences=3)
    layer.cache.page_tokens = 16
    with pytest.raises(ValueError):
        layer.branch(torch.tensor([0, 0, 1]), torch.zeros(shape, dtype=torch.int32))
    assert not moved and layer.prefix.tolist() == [0, 0, 0]


@pytest.mark.parametrize("how", ["branch", "keep"])
def test_tokens_that_were_left_behind_are_not_committed(monkeypatch, positions_of, how):
    """A step's keys and values stand behind the committed ones in the pages that its sequences had then."""
    from paper_2605_10793_amd import layer as module
    monkeypatch.setattr(module.attention, "gather", lambda *a: None)
    layer, fused, start = layer_of(sequences=2), torch.zeros(3, 8, 64), torch.tensor([0, 2, 3], dtype=torch.int32)
    layer.cache.page_tokens = 16
    layer.step(fused, start)
    if how == "branch":
        layer.branch(torch.tensor([1, 1]), layer.table)
    else:
        layer.keep(torch.tensor([], dtype=torch.int32), torch.zeros(3, dtype=torch.int32), layer.table)
    with pytest.raises(ValueError):
        layer.commit(start)
    assert layer.prefix.tolist() == [0, 0]
    layer.step(fused, start)
    layer.commit(start)
    assert layer.prefix.tolist() == [2, 1]
