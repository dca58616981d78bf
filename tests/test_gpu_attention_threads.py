"""Attention called from several threads on one stream, which PyTorch's threads share by default: each result is the one of a call by itself."""
import threading

import pytest

from test_gpu_attention import A, filled_cache, i32, randn  # noqa: F401

pytestmark = pytest.mark.gpu


def test_threads_on_one_stream_and_one_cache(A):
    """Calls that are cut into pieces, two launches each, which other threads' launches may come between."""
    import torch
    heads, width, calls, threads = 2, 128, 40, 4
    cache, table = filled_cache(A, [3000, 1700], 64, heads, width, 4, 3)
    batch = (i32([0, 3, 6]), i32([2997, 1697]), i32(table))
    q = [randn(20 + i, 6, heads * (16 if i % 2 else 4), width) for i in range(threads)]      # many rows and few
    want = [A.tree_attention(x, cache, *batch, max_query=3, max_context=3000) for x in q]
    torch.cuda.synchronize()
    got = [[] for _ in q]
    begin = threading.Barrier(threads)

    def serve(i):
        begin.wait(30)
        for _ in range(calls):
            got[i].append(A.tree_attention(q[i], cache, *batch, max_query=3, max_context=3000))

    serving = [threading.Thread(target=serve, args=(i,)) for i in range(threads)]
    for t in serving:
        t.start()
    for t in serving:
        t.join(60)
    torch.cuda.synchronize()
    for i in range(threads):
        assert len(got[i]) == calls and all(torch.equal(x, want[i]) for x in got[i])
