"""The count of a cache's pages on the host, and what the layer and the operators refuse, without a device."""
import pytest
import torch

from paper_2605_10793_amd import attention as A, binding
from paper_2605_10793_amd.layer import AttentionLayer


def test_pages_are_taken_shared_and_given_back():
    p = A.Pages(6)
    a, b = p.take(2), p.take(3)
    assert sorted(a + b) == [0, 1, 2, 3, 4] and p.left == 1
    p.share([a[0], b[0]])
    assert p.held(a[0]) == 2 and p.held(a[1]) == 1 and p.held(5) == 0
    assert p.release(a) == [a[1]] and p.left == 2
    assert p.release([a[0]]) == [a[0]] and p.left == 3
    assert set(p.take(3)) == {5, *a} and p.left == 0 and p.take(0) == []


def test_what_pages_refuse():
    p = A.Pages(3)
    a = p.take(2)
    with pytest.raises(ValueError):
        p.take(2)
    with pytest.raises(ValueError):
        p.take(-1)
    assert p.left == 1
    with pytest.raises(ValueError):
        p.share([a[0], 2])
    assert p.held(a[0]) == 1
    with pytest.raises(ValueError):
        p.release([a[0], a[1], a[1]])
    assert p.held(a[0]) == p.held(a[1]) == 1
    for bad in (-1, 3):
        with pytest.raises(ValueError):
            p.held(bad)
    assert p.release([a[0], a[1]]) == [a[0], a[1]] and p.left == 3


def test_a_page_shared_twice_in_one_call():
    p = A.Pages(1)
    a = p.take(1)
    p.share(a + a)
    assert p.held(0) == 3 and p.release(a * 2) == [] and p.release(a) == a


class Cache:
    heads, device = 2, 0


def test_a_layer_with_options_takes_no_trees():
    for options in (dict(window=5), dict(cap=30.0), dict(slopes=torch.ones(4))):
        layer = AttentionLayer(None, None, None, Cache(), torch.zeros(2, 3, dtype=torch.int32), **options)
        with pytest.raises(ValueError, match="trees"):
            layer.step(torch.zeros(4, 8, 64), torch.tensor([0, 2, 4], dtype=torch.int32), mask=torch.ones(4, dtype=torch.int64))


@pytest.mark.parametrize("prefix", [[5, 8], [0, 11]])
def test_branching_copies_the_page_that_is_begun(monkeypatch, prefix):
    """Pages of 4: which tokens the layer has moved, and the tables that it goes on with."""
    class Four(Cache):
        page_tokens = 4
    seen = []
    monkeypatch.setattr(A, "gather", lambda cache, tokens, start, table, to: seen.append([x.tolist() for x in (tokens, start, table, to)]))
    layer = AttentionLayer(None, None, None, Four(), torch.tensor([[0, 1, 2], [3, 4, 5]], dtype=torch.int32))
    layer.prefix = torch.tensor(prefix, dtype=torch.int32)
    layer.branch(torch.tensor([1, 1]), torch.tensor([[10, 11, 12], [13, 14, 15]], dtype=torch.int32))
    n = prefix[1]
    full, rest = n // 4, n % 4
    moved = [full * 4 + i if i < rest else -1 for i in range(4)]
    assert seen == [[moved * 2, [0, 4, 8], [[3, 4, 5]] * 2, [[[10, 11, 12][full]], [[13, 14, 15][full]]]]]
    assert layer.prefix.tolist() == [n, n]
    assert layer.table.tolist() == [[3, 4, 5][:full] + [10, 11, 12][full:], [3, 4, 5][:full] + [13, 14, 15][full:]]
