"""Appending where starts fall: a negative count means no tokens for that sequence, and nothing else for any other."""
import numpy as np
import pytest

from test_gpu_attention import A, i32, randn  # noqa: F401

pytestmark = pytest.mark.gpu


def falling(sequences, tokens, seed):
    """Rows of every sequence begin anywhere; about half the counts are negative, and rows may be several sequences'."""
    rng = np.random.default_rng(seed)
    return rng.integers(-20, tokens + 20, sequences + 1)


STARTS = [[0, 1000, 50, 150], [200, 20, 300], [0, 700, 0, 64, 1, 700, 699, 700], [64, 0, 64, 0, 64], [900, 900, 100, 100, 900, 100],
          *[falling(n, 500, n) for n in (2, 5, 17, 63, 64, 65, 129, 512)]]


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("start", STARTS, ids=lambda s: str(s) if isinstance(s, list) else f"{len(s) - 1} anywhere")
def test_falling_starts(A, start, bits):
    import torch
    sequences, tokens, width, page, heads = len(start) - 1, 1000, 64, 32, 2
    rng = np.random.default_rng(7)
    prefix = rng.integers(0, 130, sequences)
    columns = (tokens + 130) // page + 1
    table = rng.permutation(sequences * columns).astype(np.int32).reshape(sequences, columns)
    k, v = randn(1, tokens, heads, width), randn(2, tokens, heads, width)
    caches = [A.KVCache.empty(sequences * columns, heads, page, width, bits) for _ in range(2)]
    for c in caches:
        for x in (c.k, c.v, c.k_scale, c.v_scale):
            if x is not None:
                x.fill_(3)
    held = A.append(caches[0], k, v, i32(start), i32(prefix), i32(table), values=bits != 16)
    at = np.clip(start, 0, tokens)
    rows = np.zeros(tokens, bool)
    for b in range(sequences):             # each by itself
        lo, hi = int(at[b]), int(at[b + 1])
        if hi > lo:
            A.append(caches[1], k[lo:hi], v[lo:hi], i32([0, hi - lo]), i32(prefix[b:b + 1]), i32(table[b:b + 1]))
            rows[lo:hi] = True
    for x, y in zip((caches[0].k, caches[0].v, caches[0].k_scale, caches[0].v_scale), (caches[1].k, caches[1].v, caches[1].k_scale, caches[1].v_scale)):
        assert x is None or torch.equal(x, y)
    if bits != 16:
        whole = A.append(caches[1], k, v, i32([0, tokens]), i32([0]), i32(table.reshape(1, -1)[:, :columns]), values=True)
        pick = torch.from_numpy(rows).cuda()
        assert all(torch.equal(x[pick], y[pick]) for x, y in zip(held, whole))


@pytest.mark.parametrize("sequences", [64, 65, 200, 512, 513, 5000])
def test_rising_starts_with_empty_sequences(A, sequences):
    """Runs of empty sequences of every length between those that have tokens."""
    import torch
    rng = np.random.default_rng(sequences)
    counts = np.where(rng.random(sequences) < 0.3, rng.integers(0, 200, sequences), 0)
    counts[sequences // 3:sequences // 2] = 0
    counts[-1] = 65
    start = np.concatenate([[0], np.cumsum(counts)])
    prefix = rng.integers(0, 60, sequences)
    width, page, columns = 64, 64, 5
    table = np.arange(sequences * columns, dtype=np.int32).reshape(sequences, columns)
    cache = A.KVCache.empty(sequences * columns, 1, page, width)
    cache.k.fill_(7.0)
    cache.v.fill_(7.0)
    k, v = randn(1, start[-1], 1, width), randn(2, start[-1], 1, width)
    A.append(cache, k, v, i32(start), i32(prefix), i32(table))
    at = np.concatenate([b * columns * page + prefix[b] + np.arange(counts[b]) for b in range(sequences)])
    at = torch.from_numpy(at).cuda()
    for x, y in ((cache.k.view(-1, width), k), (cache.v.transpose(2, 3).reshape(-1, width), v)):
        want = torch.full((sequences * columns * page, width), 7.0, dtype=torch.bfloat16, device="cuda:0")
        want[at] = y[:, 0]
        assert torch.equal(x, want)


@pytest.mark.parametrize("tokens", [(1 << 29) + 5, (1 << 30) + 200, (1 << 31) - 1])
def test_more_rows_than_a_grid_counts_threads(A, tokens):
    """Rows far beyond what one launch's workgroups can be numbered by: the last of them are where they belong."""
    import torch
    width, page = 64, 64
    cache = A.KVCache.empty(6, 1, page, width)
    cache.k.fill_(7.0)
    cache.v.fill_(7.0)
    row = randn(3, 2, 1, width)
    k, v = (row[i:i + 1].expand(tokens, 1, width) for i in range(2))         # one row for all tokens
    A.append(cache, k, v, i32([0, 3, tokens - 70, tokens]), i32([0, 0, 20]), i32([[5, -1], [-1, -1], [1, 2]]))
    want = torch.full((6 * page, width), 7.0, dtype=torch.bfloat16, device="cuda:0")
    for first, last in ((5 * page, 5 * page + 3), (page + 20, page + 90)):
        want[first:last] = row[0]
    assert torch.equal(cache.k.view(-1, width), want)
    for first, last in ((5 * page, 5 * page + 3), (page + 20, page + 90)):
        want[first:last] = row[1]
    assert torch.equal(cache.v.transpose(2, 3).reshape(-1, width), want)
