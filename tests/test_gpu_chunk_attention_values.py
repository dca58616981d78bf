"""Chunk attention and moved tokens: what is not finite, rows anywhere, shared pages, far pages, streams, threads, graphs; the layer that runs them together."""
import math
import threading

import pytest
import torch

from attention_reference import attend, close, seen_of
from test_gpu_chunk_attention import filled

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def randn(seed, *shape):
    return torch.randn(*shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(seed)).to(torch.bfloat16)


def held_of(cache, row, n):
    """What a cache holds of a sequence's n tokens, 64 bits, [n, heads, width] each, and what its sums are made of (codes)."""
    pages = row.long().cpu()[:(n + cache.page_tokens - 1) // cache.page_tokens]
    both, sizes = [], []
    for side, (pool, scale) in enumerate(((cache.k, cache.k_scale), (cache.v, cache.v_scale))):
        x = pool.cpu()[pages]
        x = x.transpose(2, 3) if side else x
        if cache.bits == 4:
            x = torch.cat([x & 15, x >> 4], -1)
        x = x.double()
        if cache.bits != 16:
            pair = scale.cpu()[pages].double()
            x = x * pair[..., :1] + pair[..., 1:]
            sizes.append((pair[..., 1].abs() + 383 * pair[..., 0].abs()).transpose(1, 2).reshape(-1, cache.heads)[:n])
        both.append(x.transpose(1, 2).reshape(-1, cache.heads, cache.width)[:n])
    return both, sizes or None


@pytest.mark.parametrize("n", [3, 40, 100])
@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_what_a_token_does_not_see_has_no_influence(n, value, cap):
    from paper_2605_10793_amd import attention as A
    a, heads, kv, width, page = 150, 4, 2, 64, 32
    cache, table, _ = filled(16, kv, page, width, [a + n], seed=n)
    q, start, prefix, table = randn(1, n, heads, width), i32([0, n]), i32([a]), table.to(DEV)
    for window in (0, 60):
        clean = A.chunk_attention(q, cache, start, prefix, table, window=window, cap=cap)
        t = a + n - 2                       # a new token before the last: seen by itself and the last
        page_at, slot = int(table[0, t // page]), t % page
        keep = cache.k[page_at, 0, slot].clone(), cache.v[page_at, 1, :, slot].clone()
        cache.k[page_at, 0, slot], cache.v[page_at, 1, :, slot] = value, value
        got = A.chunk_attention(q, cache, start, prefix, table, window=window, cap=cap)
        assert torch.equal(got[:n - 2], clean[:n - 2])
        assert not bool(torch.isfinite(got[n - 2:, 2:]).any())
        cache.k[page_at, 0, slot], cache.v[page_at, 1, :, slot] = keep
        if window:                          # and one that only the first ones' windows reach
            t = a - 50
            page_at, slot = int(table[0, t // page]), t % page
            keep = cache.k[page_at, :, slot].clone(), cache.v[page_at, :, :, slot].clone()
            cache.k[page_at, :, slot], cache.v[page_at, :, :, slot] = value, value
            got = A.chunk_attention(q, cache, start, prefix, table, window=window, cap=cap)
            behind = t + window - a         # the first new token that does not see it
            assert torch.equal(got[behind:], clean[behind:]) and not bool(torch.isfinite(got[:min(behind, n)]).all())
            cache.k[page_at, :, slot], cache.v[page_at, :, :, slot] = keep


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("n", [2, 50])
def test_rows_anywhere(bits, n):
    from paper_2605_10793_amd import attention as A
    cache, table, _ = filled(bits, 2, 64, 128, [70 + n, 9 + n], seed=bits)
    q, start, prefix, table = randn(2, 2 * n, 8, 128), i32([0, n, 2 * n]), i32([70, 9]), table.to(DEV)
    want = A.chunk_attention(q, cache, start, prefix, table, max_query=n)
    wide = torch.zeros(2 * n, 13, 131, dtype=torch.bfloat16, device=DEV)
    moved, out = wide[:, 2:10, 1:129], torch.zeros(8, 2 * n, 129, dtype=torch.bfloat16, device=DEV)[..., :128].transpose(0, 1)
    moved.copy_(q)
    A.chunk_attention(moved, cache, start, prefix, table, max_query=n, out=out)
    assert torch.equal(out, want)
    A.chunk_attention(q, cache, start, prefix, table, max_query=n, out=q)           # over the queries
    assert torch.equal(q, want)


def test_shared_pages_and_an_order_of_pages():
    """Sequences that have pages in common get what they would with copies of them."""
    from paper_2605_10793_amd import attention as A
    cache, table, _ = filled(16, 2, 16, 64, [64 + 5, 64 + 5], seed=3)
    table[1, :4] = table[0, :4]
    q, start, prefix = randn(3, 10, 4, 64), i32([0, 5, 10]), i32([64, 64])
    got = A.chunk_attention(q, cache, start, prefix, table.to(DEV), max_query=5)
    alone = [A.chunk_attention(q[5 * b:5 * b + 5], cache, i32([0, 5]), i32([64]), table[b:b + 1].to(DEV), max_query=5) for b in range(2)]
    assert torch.equal(got, torch.cat(alone))


def test_pages_and_rows_far_apart():
    """Offsets beyond 31 and 32 bits: pages at the end of a pool of 5 GiB a side; packed rows 8 MiB apart."""
    from paper_2605_10793_amd import attention as A
    small, table, held = filled(16, 8, 64, 128, [200], seed=4, spare=0)
    pages = 40960
    big = A.KVCache.empty(pages, 8, 64, 128, 16, DEV)
    far = [pages - 1 - 7 * i for i in range(small.pages)]
    for i, p in enumerate(far):
        big.k[p], big.v[p] = small.k[i], small.v[i]
    q, start, prefix = randn(4, 9, 16, 128), i32([0, 9]), i32([191])
    there = torch.tensor(far, dtype=torch.int32)[table.long()].to(DEV)
    for m in (9, 100):
        assert torch.equal(A.chunk_attention(q, big, start, prefix, there, max_query=m), A.chunk_attention(q, small, start, prefix, table.to(DEV), max_query=m))
    to = i32([[0, 1, 2, 3]])
    A.gather(big, torch.arange(200, dtype=torch.int32, device=DEV), i32([0, 200]), there, to)
    for c in range(4):
        n = min(64, 200 - 64 * c)
        assert torch.equal(big.k[c, :, :n], big.k[int(there[0, c]), :, :n]) and torch.equal(big.v[c, :, :, :n], big.v[int(there[0, c]), :, :, :n])
    del big
    n, apart = 300, (1 << 22) - 64
    flat = torch.empty(n * apart, dtype=torch.bfloat16, device=DEV).view(n, apart)
    parts = [flat[:, 256 * i:256 * i + 256].view(n, 2, 128) for i in range(4)]
    for i, x in enumerate(parts):
        x.copy_(randn(10 + i, n, 2, 128))
    start = i32([0, n])
    out, lse = A.attention(*parts[:3], start, lse=True)
    grads = A.attention_backward(*parts[:3], out, lse, parts[3], start)
    near = [x.contiguous() for x in parts]
    want, sums = A.attention(*near[:3], start, lse=True)
    assert torch.equal(out, want) and torch.equal(lse, sums)
    for x, y in zip(grads, A.attention_backward(*near[:3], want, sums, near[3], start)):
        assert torch.equal(x, y)


def test_graphs_streams_and_threads():
    """Two captured graphs, eager calls between their replays, a side stream, two threads on one stream: each call's own result."""
    from paper_2605_10793_amd import attention as A
    cache, table, _ = filled(8, 2, 64, 128, [3000, 2500, 700], seed=5)
    table, start, prefix = table.to(DEV), i32([0, 20, 40, 60]), i32([2980, 2480, 680])
    inputs = [randn(20 + i, 60, 8, 128) for i in range(4)]
    call = lambda x, **o: A.chunk_attention(x, cache, start, prefix, table, max_query=20, **o)  # noqa: E731
    want = [call(x) for x in inputs]
    windowed = [call(x, window=999) for x in inputs]
    torch.cuda.synchronize()
    x, y = inputs[0].clone(), inputs[0].clone()
    one, two = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(one):
        a = call(x)
    with torch.cuda.graph(two):
        b = call(y, window=999)
    for i in range(4):
        x.copy_(inputs[i])
        y.copy_(inputs[3 - i])
        one.replay()
        two.replay()
        eager = call(inputs[i])
        torch.cuda.synchronize()
        assert torch.equal(a, want[i]) and torch.equal(b, windowed[3 - i]) and torch.equal(eager, want[i])
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = call(inputs[1])
    here = call(inputs[2])
    torch.cuda.synchronize()
    assert torch.equal(got, want[1]) and torch.equal(here, want[2])
    found = {}

    def serve(i):
        with torch.no_grad():
            found[i] = [call(inputs[i]) for _ in range(5)]

    threads = [threading.Thread(target=serve, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    torch.cuda.synchronize()
    assert sorted(found) == [0, 1, 2, 3]
    for i, results in found.items():
        assert all(torch.equal(r, want[i]) for r in results)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("window, cap, biased", [(0, 0.0, False), (100, 30.0, True)])
def test_a_layer_serves_prompts_tokens_and_branches(bits, window, cap, biased):
    """Prompts in one chunk, single tokens, a branch into other pages, a sequence that drops tokens: every step's outputs against 64 bits over what the cache holds."""
    from paper_2605_10793_amd import attention as A
    from paper_2605_10793_amd.layer import AttentionLayer
    heads, kv, width, page, B, columns = 4, 2, 64, 16, 3, 16
    pages = A.Pages(2 * B * columns)
    held = [pages.take(columns) for _ in range(B)]
    cache = A.KVCache.empty(2 * B * columns, kv, page, width, bits, DEV)
    weight = torch.ones(width, dtype=torch.bfloat16, device=DEV)
    slopes = torch.tensor([0.5, 0.1, 0.02, 0.0], device=DEV) if biased else None
    layer = AttentionLayer(A.Rotary(width, device=DEV), weight, weight, cache, i32(held), window=window, cap=cap, slopes=slopes)
    spread = 0.3 + torch.rand(1, heads + 2 * kv, width, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    lengths = [0] * B

    def step(counts, seed):
        nonlocal lengths
        tokens, start = sum(counts), [sum(counts[:b]) for b in range(B + 1)]
        fused = (randn(seed, tokens, heads + 2 * kv, width) * spread).to(torch.bfloat16)
        out = layer.step(fused, i32(start), max_query=max(counts))
        rows = torch.cat([torch.arange(n) + lengths[b] for b, n in enumerate(counts)]).to(DEV)
        q, _ = A.qk_norm_rotary(layer.plan, fused[:, :heads], fused[:, heads:heads + kv], weight, weight, rows)
        for b, n in enumerate(counts):
            mine = slice(start[b], start[b + 1])
            both, sizes = held_of(cache, layer.table[b], lengths[b] + n)
            want = attend(q[mine].cpu(), *both, seen_of(n, None, None, window, lengths[b]), torch.arange(lengths[b], lengths[b] + n), width ** -0.5, cap,
                          None if slopes is None else slopes.cpu(), sizes=sizes)
            close(out[mine], want["out"], want["out_tol"], f"sequence {b}")
        layer.commit(i32(start))
        lengths = [m + n for m, n in zip(lengths, counts)]
        assert layer.prefix.tolist() == lengths

    step([130, 70, 90], 1)
    step([1, 1, 1], 2)
    parents = [1, 1, 0]
    shared = [held[p][:lengths[p] // page] for p in parents]
    for x in shared:
        pages.share(x)
    fresh = [x + pages.take(columns - len(x)) for x in shared]
    for x in held:
        pages.release(x)
    layer.branch(torch.tensor(parents, device=DEV), i32(fresh))
    lengths = [lengths[p] for p in parents]
    assert layer.table.tolist() == fresh and pages.left == 2 * B * columns - len({p for x in fresh for p in x})
    step([1, 2, 65], 3)
    step([1, 1, 1], 4)
    old = [held_of(cache, layer.table[b], n)[0] for b, n in enumerate(lengths)]
    kept = [torch.arange(0, n, 2) for n in lengths]
    to = i32([pages.take(8) for _ in range(B)])
    layer.keep(torch.cat(kept).to(torch.int32).to(DEV), i32([sum(len(x) for x in kept[:b]) for b in range(B + 1)]), to)
    lengths = [len(x) for x in kept]
    assert layer.prefix.tolist() == lengths
    for b in range(B):
        for x, y in zip(old[b], held_of(cache, layer.table[b], lengths[b])[0]):
            assert torch.equal(x[kept[b]], y)
    step([2, 1, 3], 5)


def test_a_layer_trains_on_packed_sequences():
    """Norms, positions and attention, forward and back: the operators one by one give the same, and the loss moves as its gradients say."""
    from paper_2605_10793_amd import attention as A
    from paper_2605_10793_amd.layer import AttentionLayer
    heads, kv, width = 4, 2, 64
    weight = (1 + 0.1 * randn(7, width).float()).to(torch.bfloat16)
    cache = A.KVCache.empty(1, kv, 16, width, 16, DEV)
    layer = AttentionLayer(A.Rotary(width, device=DEV), weight, weight, cache, i32([[0]]), cap=20.0)
    fused, start = randn(8, 90, heads + 2 * kv, width), i32([3, 40, 85])
    grad = randn(9, 90, heads, width)
    out = layer.packed(fused, start)
    dfused, dq_weight, dk_weight = layer.packed_gradients(grad)
    positions = torch.zeros(90, dtype=torch.int64, device=DEV)
    for a, b in ((3, 40), (40, 85)):
        positions[a:b] = torch.arange(b - a, device=DEV)
    positions[:3], positions[85:] = layer._trained[5][:3], layer._trained[5][85:]
    q, k = A.qk_norm_rotary(layer.plan, fused[:, :heads], fused[:, heads:heads + kv], weight, weight, positions)
    want, lse = A.attention(q, k, fused[:, heads + kv:], start, lse=True, cap=20.0)
    assert torch.equal(out, want) and not out[:3].any() and not out[85:].any()
    dq, dk, dv = A.attention_backward(q, k, fused[:, heads + kv:], want, lse, grad, start, cap=20.0)
    dq, dk, a, b = A.qk_norm_rotary_backward(layer.plan, fused[:, :heads], fused[:, heads:heads + kv], weight, weight, positions, dq, dk)
    assert torch.equal(dfused, torch.cat([dq, dk, dv], 1)) and torch.equal(a, dq_weight) and torch.equal(b, dk_weight)
    assert not dfused[:3].any() and not dfused[85:].any() and bool(torch.isfinite(dfused).all())
