"""Chunk attention where starts fall: a negative count means no tokens for that sequence, and nothing else for any other."""
import pytest
import torch

from attention_reference import attend, close, seen_of
from test_gpu_chunk_attention import filled

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def check(bits, page, width, heads, kv, start, tokens, committed, given, cap=0.0, max_query=None, seed=0):
    """Rows of sequences against 64 bits; rows without a result as they were in a `given` tensor, zeros in a new one."""
    from paper_2605_10793_amd import attention as A
    edges = [min(max(x, 0), tokens) for x in start]
    counts = [max(0, y - x) for x, y in zip(edges, edges[1:])]
    cache, table, held = filled(bits, kv, page, width, [a + n for a, n in zip(committed, counts)], seed)
    q = torch.randn(tokens, heads, width, generator=torch.Generator().manual_seed(seed + 1)).to(torch.bfloat16)
    out = torch.full_like(q, 7).to(DEV) if given else None
    got = A.chunk_attention(q.to(DEV), cache, torch.tensor(start, dtype=torch.int32, device=DEV), torch.tensor(committed, dtype=torch.int32, device=DEV),
                            table.to(DEV), cap=cap, max_query=max_query or max(counts), max_context=max(a + n for a, n in zip(committed, counts)), out=out)
    without = torch.ones(tokens, dtype=torch.bool)
    for b, (x, a, n) in enumerate(zip(edges, committed, counts)):
        m = min(n, max_query or n)
        assert bool(without[x:x + n].all())          # (each row one sequence's)
        if not n:
            continue
        without[x:x + m] = False
        want = attend(q[x:x + m], *held[b][0], seen_of(n, None, None, 0, a)[:m], torch.arange(a, a + m), width ** -0.5, cap, sizes=held[b][1])
        close(got[x:x + m], want["out"], want["out_tol"], f"sequence {b}")
    assert bool((got[without.to(DEV)] == (7 if given else 0)).all())


def backwards(pieces, size):
    """Sequences of `size` rows whose rows lie one behind the other from the last to the first, and sequences of none between them."""
    return [x for i in reversed(range(pieces)) for x in (i * size, (i + 1) * size)]


# starts, rows of the call, committed tokens
FALLING = [([0, 200, 0, 0], 200, [30, 0, 9]),                                   # padded by zeros
           ([150, 300, 0, 150, 100], 320, [10, 70, 0, 64]),                     # the first rows are a later sequence's
           ([40, 10, 140, 140, 0, 9], 150, [5, 33, 0, 90, 1]),                  # falls at the front and between
           ([-5, 90, 400, 230, -9, -1], 240, [0, 64, 3, 0, 20]),                # beyond the rows at both ends
           ([300, 200, 100, 0], 300, [1, 2, 3]),                                # falls throughout
           (backwards(5, 70), 350, [(i * 37) % 90 for i in range(9)])]


FORMATS = [(16, 64, 128), (8, 32, 64), (4, 16, 128)]


@pytest.mark.parametrize("bits, page, width", FORMATS)
@pytest.mark.parametrize("start, tokens, committed", FALLING, ids=lambda x: str(x) if isinstance(x, list) else None)
def test_row_tiles_of_every_sequence(bits, page, width, start, tokens, committed):
    """Several row tiles and no runs."""
    check(bits, page, width, 8, 2, start, tokens, committed, True, max_query=400, seed=tokens)


def test_two_tiles_of_few_rows():
    check(8, 64, 128, 8, 2, [0, 7, 0, 0], 7, [70, 5, 5], True, cap=20.0)
    check(8, 64, 128, 8, 2, backwards(20, 7), 145, [(i * 37) % 90 for i in range(39)], True, cap=20.0)


@pytest.mark.parametrize("pieces", [32, 33, 100, 256])
def test_many_sequences(pieces):
    """Around the numbers of sequences that a wavefront looks at together, up to the most whose starts may fall."""
    check(16, 16, 64, 4, 1, backwards(pieces, 33), 33 * pieces, [i % 3 for i in range(2 * pieces - 1)], True, max_query=100)
    check(4, 16, 64, 4, 1, [33 * pieces] * 2 + backwards(pieces, 33)[:-2], 33 * pieces, [i % 3 for i in range(2 * pieces - 1)], True, max_query=20)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("size", [1, 90])
def test_runs(bits, size):
    """Contexts that are cut into runs."""
    check(bits, 64, 128, 8, 2, [0, size, 0, 0], size, [3000, 9, 0], True)
    check(bits, 64, 128, 8, 2, backwards(3, size), 3 * size, [2500, 0, 900, 4, 3000], True)


@pytest.mark.parametrize("bits, page, width", FORMATS)
@pytest.mark.parametrize("start, tokens, committed", [*FALLING, ([0, 1, 2, 0, 0], 2, [7, 100, 3, 4]), ([3, 4, 1, 2, 0, 1], 6, [7, 0, 3, 4, 90])],
                         ids=lambda x: str(x) if isinstance(x, list) else None)
def test_rows_without_a_result_are_zeros(bits, page, width, start, tokens, committed):
    """In a new tensor; no others are."""
    check(bits, page, width, 8, 2, start, tokens, committed, False, max_query=400 if tokens > 9 else None, seed=tokens)


@pytest.mark.parametrize("bits, committed", [(16, 10), (16, 3000), (8, 3000), (4, 40)])
@pytest.mark.parametrize("size, max_query", [(1, 1), (3, 2), (50, 40)])
def test_many_rows_without_a_result(bits, committed, size, max_query):
    """Behind the sequences and before them, beyond the most new tokens, with runs and without."""
    for start, tokens in (([0, size, 2 * size], 4001), ([4000 - size, 4000, 0], 4000), ([1700, 1700 + size, 0], 1701 + size), ([900, 900, 900 + size], 4000)):
        check(bits, 64, 128, 8, 2, start, tokens, [committed, 20], False, max_query=max_query)


@pytest.mark.parametrize("sequences", [511, 512, 513, 700])
def test_rows_without_a_result_among_many_sequences(sequences):
    """Around the most sequences whose starts may fall: sequences of none, of more than have results, rows before and behind them."""
    counts = [(i * 7) % 4 if i % 5 else 0 for i in range(sequences)]
    start = [37 + sum(counts[:b]) for b in range(sequences + 1)]
    check(16, 16, 64, 2, 1, start, start[-1] + 70, [i % 3 for i in range(sequences)], False, max_query=2)


def test_rows_without_a_result_at_any_strides(monkeypatch):
    from paper_2605_10793_amd import attention as A
    monkeypatch.setattr(A, "_like", lambda x: torch.full((x.shape[1], x.shape[0], x.shape[2] + 1), 7, dtype=x.dtype, device=x.device)[..., 1:].transpose(0, 1))
    check(16, 64, 64, 4, 2, [5, 9, 0], 300, [30, 0], False, max_query=3)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("max_query, context", [(4, 40), (4, 2000), (200, 250)])
def test_a_captured_call_of_batches_of_any_size(bits, max_query, context):
    """One graph, replayed with other starts, prefixes and queries, the batch padded by sequences of none and rows of no sequence."""
    from paper_2605_10793_amd import attention as A
    sequences, tokens = 6, 3 * max_query
    cache, table, _ = filled(bits, 2, 64, 128, [context] * sequences, seed=1)
    table = table.to(DEV)
    q, start, prefix = (torch.zeros(s, dtype=t, device=DEV) for s, t in (((tokens, 8, 128), torch.bfloat16), ((sequences + 1,), torch.int32), ((sequences,), torch.int32)))
    call = lambda q, s, p: A.chunk_attention(q, cache, s, p, table[:p.shape[0]], max_query=max_query, max_context=context)  # noqa: E731
    call(q, start, prefix)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(q, start, prefix)
    g = torch.Generator().manual_seed(2)
    for counts in ([max_query] * 3, [1], [2, 0, max_query, 1], [], [max_query, 1, 1, 1, 1, 1], [0, max_query]):
        n, total = len(counts), sum(counts)
        edges = [sum(counts[:b]) for b in range(n + 1)]
        q.copy_(torch.randn(tokens, 8, 128, generator=g))
        start.copy_(torch.tensor(edges + [0] * (sequences - n)))
        prefix.copy_(torch.tensor([(37 * b + 11) % (context - max_query) for b in range(sequences)]))
        graph.replay()
        eager = call(q, start, prefix)
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and not out[total:].any()
        for b, (x, y) in enumerate(zip(edges, edges[1:])):          # each by itself: two results, off by two roundings of 2^-8 each at most
            if y > x:
                own = A.chunk_attention(q[x:y], cache, torch.tensor([0, y - x], dtype=torch.int32, device=DEV), prefix[b:b + 1].clone(), table[b:b + 1],
                                        max_query=max_query, max_context=context)
                assert float((own.double() - out[x:y].double()).norm()) <= 4 * 2.0 ** -8 * float(own.double().norm())
