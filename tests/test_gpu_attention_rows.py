"""Rows of attention's result that no token has a result for."""
import pytest

from test_gpu_attention import A, filled_cache, i32, randn  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("counts,max_query", [([100], 64), ([100, 3], 64), ([5, 70, 0, 66], 64), ([9], 4), ([3, 3, 1], 2)])
def test_rows_beyond_max_query_are_zeros_in_a_new_tensor(A, counts, max_query):
    """Not what the allocator's block held; the others are what they are by themselves."""
    import torch
    heads, width = 1, 64
    lengths = [80 + n for n in counts]
    cache, table = filled_cache(A, lengths, 32, heads, width, 16, 5)
    q = randn(3, sum(counts), 2, width)
    start = [sum(counts[:b]) for b in range(len(counts) + 1)]
    batch = (i32(start), i32([80] * len(counts)), i32(table))
    more = {} if max_query == 64 else dict(max_query=max_query)
    want = A.tree_attention(q, cache, *batch, out=torch.zeros_like(q), **more)
    for _ in range(3):
        poison = torch.full_like(q, float("nan"))
        del poison
        got = A.tree_attention(q, cache, *batch, **more)
        assert torch.equal(got, want)
        assert all(torch.all(got[start[b] + max_query:start[b + 1]] == 0) for b in range(len(counts)))
        del got
