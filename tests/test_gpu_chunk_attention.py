"""Attention of chunks of new tokens over the paged cache, and moves of its tokens, against 64 bits: formats, pages, lengths, masks, layouts."""
import pytest
import torch

from attention_reference import attend, close, seen_of
from test_gpu_packed_attention import lists

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def filled(bits, heads, page, width, lengths, seed, spare=2, holes=()):
    """A cache of sequences of `lengths` tokens in mixed pages, its table, and what it holds of each sequence in 64 bits."""
    from paper_2605_10793_amd import attention as A
    g = torch.Generator().manual_seed(seed)
    need = [(n + page - 1) // page for n in lengths]
    columns, pages = max(max(need), 1), sum(need) + spare
    order = torch.randperm(pages, generator=g).tolist()
    table, at = torch.full((len(lengths), columns), -1, dtype=torch.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    cache = A.KVCache.empty(pages, heads, page, width, bits, DEV)
    for x in (cache.k, cache.v, cache.k_scale, cache.v_scale):      # what no token was put into holds NaN, or codes and pairs of anything
        if x is not None:
            x.fill_(float("nan") if x.is_floating_point() else 77)
    tokens = sum(lengths)
    rows = torch.randn(tokens, 2 * heads, width, generator=g) * torch.exp(0.5 * torch.randn(2 * heads, width, generator=g)) + 0.2
    rows = rows.to(torch.bfloat16).to(DEV)
    start = torch.tensor([sum(lengths[:b]) for b in range(len(lengths) + 1)], dtype=torch.int32, device=DEV)
    zero = torch.zeros(len(lengths), dtype=torch.int32, device=DEV)
    A.append(cache, rows[:, :heads], rows[:, heads:], start, zero, table.to(DEV))
    held, sizes = [], []
    for b, n in enumerate(lengths):
        both = []
        for side in (0, 1):
            pool, scale = (cache.k, cache.k_scale) if side == 0 else (cache.v, cache.v_scale)
            pool = pool.cpu()
            if side:
                pool = pool.transpose(2, 3)
            if bits == 4:
                pool = torch.cat([pool & 15, pool >> 4], -1)
            pool = pool.double()
            if bits != 16:
                pool = pool * scale.cpu()[..., :1].double() + scale.cpu()[..., 1:].double()
            own = table[b, :need[b]].long()
            both.append(pool[own].transpose(1, 2).reshape(-1, heads, width)[:n])
        held.append(both)
        if bits != 16:
            pairs = [x.cpu()[own].transpose(1, 2).reshape(-1, heads, 2)[:n].abs() for x in (cache.k_scale, cache.v_scale)]
            sizes.append([x[..., 1] + (128 + 255) * x[..., 0] for x in pairs])
    for b, column in holes:
        table[b, column] = -1
    return cache, table, list(zip(held, sizes if sizes else [None] * len(held)))


def check(bits, page, width, committed, counts, heads, kv, kind="causal", window=0, cap=0.0, biased=False, seed=0, holes=(), max_query=None, closer=False,
          scale=None):
    from paper_2605_10793_amd import attention as A
    lengths = [a + n for a, n in zip(committed, counts)]
    cache, table, held = filled(bits, kv, page, width, lengths, seed, holes=holes)
    g = torch.Generator().manual_seed(seed + 1)
    tokens = sum(counts)
    q = torch.randn(tokens + 3, heads, width, generator=g).to(torch.bfloat16)
    first, last = lists(counts, kind)
    if first is not None:      # bounds in tokens of the sequence
        first = [x + (a if kind != "prefix" else 0) for x, a in zip(first, [a for a, n in zip(committed, counts) for _ in range(n)])]
        last = [x + a for x, a in zip(last, [a for a, n in zip(committed, counts) for _ in range(n)])]
    slopes = torch.exp2(-8 * (1 + torch.arange(heads, dtype=torch.float32)) / heads) if biased else None
    pad = lambda x: None if x is None else torch.tensor(x + [0] * 3, dtype=torch.int32, device=DEV)
    start = torch.tensor([sum(counts[:b]) for b in range(len(counts) + 1)], dtype=torch.int32, device=DEV)
    prefix = torch.tensor(committed, dtype=torch.int32, device=DEV)
    options = dict(first=pad(first), last=pad(last), window=window, cap=cap, slopes=None if slopes is None else slopes.to(DEV), scale=scale)
    if closer:
        options.update(max_query=max(counts), max_context=max(lengths))
    if max_query is not None:
        options.update(max_query=max_query)
    out = A.chunk_attention(q.to(DEV), cache, start, prefix, table.to(DEV), **options)
    assert not out[tokens:].any()
    given = torch.full_like(q.to(DEV), 7)
    A.chunk_attention(q.to(DEV), cache, start, prefix, table.to(DEV), out=given, **options)
    assert bool((given[tokens:] == 7).all())
    at = 0
    for b, (a, n) in enumerate(zip(committed, counts)):
        m = n if max_query is None else min(n, max_query)
        mine = slice(at, at + n)
        seen = seen_of(n, first and first[mine], last and last[mine], window, a)[:m]
        for hb, column in holes:
            if hb == b:
                seen = seen & ~((torch.arange(a + n) // page) == column)[None]
        want = attend(q[at:at + m], *held[b][0], seen, torch.arange(a, a + m), width ** -0.5 if scale is None else scale, cap, slopes, sizes=held[b][1])
        close(out[at:at + m], want["out"], want["out_tol"], f"sequence {b}")
        assert torch.equal(given[at:at + m], out[at:at + m])
        assert not out[at + m:at + n].any() and bool((given[at + m:at + n] == 7).all())
        at += n


FORMATS = [(16, 64, 128), (16, 16, 64), (8, 32, 128), (8, 64, 64), (4, 128, 128), (4, 16, 64), (16, 256, 64)]


@pytest.mark.parametrize("bits, page, width", FORMATS)
@pytest.mark.parametrize("closer", [False, True])
def test_one_token(bits, page, width, closer):
    check(bits, page, width, [0, 1, 63, 64, 500, 777], [1] * 6, 8, 2, seed=bits + page, closer=closer)


@pytest.mark.parametrize("bits, page, width", FORMATS)
@pytest.mark.parametrize("kind, window, cap, biased", [("causal", 0, 0.0, False), ("causal", 100, 0.0, False), ("prefix", 0, 30.0, False), ("causal", 70, 0.0, True),
                                                       ("holes", 0, 0.0, False), ("both", 0, 5.0, True)])
def test_few(bits, page, width, kind, window, cap, biased):
    check(bits, page, width, [300, 0, 64, 901], [3, 7, 1, 5], 4, 1, kind=kind, window=window, cap=cap, biased=biased, seed=bits + page, closer=True)


@pytest.mark.parametrize("bits, page, width", FORMATS)
@pytest.mark.parametrize("kind, window, cap, biased", [("causal", 0, 0.0, False), ("causal", 100, 0.0, False), ("prefix", 0, 30.0, False), ("causal", 0, 0.0, True),
                                                       ("documents", 0, 0.0, False), ("far", 0, 4.0, True)])
def test_chunks(bits, page, width, kind, window, cap, biased):
    check(bits, page, width, [130, 0, 700], [150, 70, 33], 8, 2, kind=kind, window=window, cap=cap, biased=biased, seed=bits + page + 1, closer=window > 0)


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_split_long(bits):
    check(bits, 64, 128, [6000], [1], 8, 2, seed=5, closer=True)
    check(bits, 64, 128, [5000], [60], 4, 1, seed=6, closer=True)
    check(bits, 64, 64, [3000, 20], [200, 9], 2, 2, seed=7, closer=True, window=1500)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("n", [2, 90])
def test_missing_pages(bits, n):
    check(bits, 32, 64, [200, 400], [n, n], 4, 2, seed=8, holes=((0, 1), (0, 0), (1, 5)))
    check(bits, 64, 128, [200, 400], [n, n], 4, 2, seed=9, holes=((1, 0), (1, 4)))


@pytest.mark.parametrize("n", [40, 5])
def test_more_than_max_query(n):
    check(16, 64, 128, [100, 7, 0], [n, n + 30, 2], 4, 2, seed=10, max_query=n)


@pytest.mark.parametrize("heads, kv", [(1, 1), (5, 1), (16, 16), (64, 1)])
@pytest.mark.parametrize("n", [1, 65])
def test_head_layouts(heads, kv, n):
    check(16, 64, 128, [150], [n], heads, kv, seed=heads)
    check(4, 64, 128, [150], [n], heads, kv, seed=heads)


def test_scales():
    check(16, 64, 64, [100], [70], 2, 1, seed=12, scale=-0.3)
    check(8, 64, 64, [100], [3], 2, 1, seed=13, scale=-0.3, cap=10.0)
    check(4, 64, 64, [100], [70], 2, 1, seed=13, scale=-0.3, cap=10.0)


@pytest.mark.parametrize("bits, page, width", [(16, 64, 128), (8, 32, 128), (4, 16, 64)])
@pytest.mark.parametrize("counts, heads", [([1] * 40 + [230] + [1] * 30 + [65, 0, 3], 8), ([1, 2, 0, 1] * 16, 4), ([66] * 63, 4), ([130] * 5, 4), ([17] * 65, 2)])
def test_prompts_among_tokens(bits, page, width, counts, heads):
    """Sequences of a call that bring very different numbers of tokens, over little that is committed and with limits that the table and q give."""
    committed = [(i * 53) % 130 for i in range(len(counts))]
    check(bits, page, width, committed, counts, heads, 2, seed=len(counts) + bits, closer=heads == 4)
    check(bits, page, width, committed, counts, heads, 2, seed=len(counts) + bits, max_query=40)


@pytest.mark.parametrize("bits, page, width", FORMATS)
@pytest.mark.parametrize("what", ["fork", "keep", "all", "shift"])
def test_gather(bits, page, width, what):
    from paper_2605_10793_amd import attention as A
    lengths = [1, 130, 64, 0, 517]
    cache, table, held = filled(bits, 3, page, width, lengths, seed=page, spare=60)
    used = {int(x) for x in table.flatten() if x >= 0}
    free = [p for p in range(cache.pages) if p not in used]
    g = torch.Generator().manual_seed(4)
    if what == "fork":
        pick = [torch.arange(n // page * page, n) for n in lengths]
    elif what == "keep":
        pick = [torch.randperm(n, generator=g)[:n * 3 // 4] for n in lengths]
    elif what == "all":
        pick = [torch.arange(n) for n in lengths]
    else:
        pick = [torch.arange(min(n, 3), n) for n in lengths]
    columns = max(1, max((len(p) + page - 1) // page for p in pick))
    to_table = torch.full((5, columns), -1, dtype=torch.int32)
    for b, p in enumerate(pick):
        n = (len(p) + page - 1) // page
        to_table[b, :n] = torch.tensor([free.pop() for _ in range(n)], dtype=torch.int32)
    old = [None if x is None else x.cpu().clone() for x in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    tokens = torch.cat(pick).to(torch.int32)
    start = torch.tensor([sum(len(p) for p in pick[:b]) for b in range(6)], dtype=torch.int32)
    A.gather(cache, tokens.to(DEV), start.to(DEV), table.to(DEV), to_table.to(DEV))
    for side, (x, y) in enumerate(zip(old, (cache.k, cache.v, cache.k_scale, cache.v_scale))):
        if x is None:
            continue
        want = x.clone()
        for b, p in enumerate(pick):
            for i, t in enumerate(p.tolist()):
                f, fs, to, ts = int(table[b, t // page]), t % page, int(to_table[b, i // page]), i % page
                if side == 1:
                    want[to, :, :, ts] = x[f, :, :, fs]
                else:
                    want[to, :, ts] = x[f, :, fs]
        assert torch.equal(want.view(torch.uint8), y.cpu().view(torch.uint8))


@pytest.mark.parametrize("n", [1, 63, 64, 65, 4032, 4096])
def test_gather_counts_of_sequences(n):
    """Around those where a part's sequence is found in one read more: every sequence is moved, the last one too."""
    from paper_2605_10793_amd import attention as A
    lengths = [1 + i % 3 for i in range(n - 1)] + [70]
    cache = A.KVCache.empty(2 * (n + 1), 1, 64, 64, 16, DEV)
    cache.k.copy_(torch.arange(cache.k.numel(), dtype=torch.int32, device=DEV).view(torch.int16)[:cache.k.numel()].view(cache.k.shape).view(torch.bfloat16))
    cache.v.zero_()
    table = torch.full((n, 2), -1, dtype=torch.int32)
    table[:, 0] = torch.arange(n, dtype=torch.int32)
    table[n - 1, 1] = n
    to_table = torch.where(table < 0, table, table + n + 1)
    tokens = torch.cat([torch.arange(m, dtype=torch.int32).flip(0) for m in lengths])
    start = torch.tensor([0] + lengths).cumsum(0).to(torch.int32)
    want = cache.k.cpu().view(torch.int16).clone()
    for b, m in enumerate(lengths):
        for i in range(m):
            t = m - 1 - i
            want[to_table[b, i // 64], 0, i % 64] = want[table[b, t // 64], 0, t % 64]
    A.gather(cache, tokens.to(DEV), start.to(DEV), table.to(DEV), to_table.to(DEV))
    assert torch.equal(want, cache.k.cpu().view(torch.int16))


def test_gather_without_places():
    """Tokens out of a table's reach, and pages that are none, are not moved."""
    from paper_2605_10793_amd import attention as A
    cache, table, _ = filled(16, 2, 16, 64, [40, 40], seed=3, spare=8)
    used = {int(x) for x in table.flatten() if x >= 0}
    free = [p for p in range(cache.pages) if p not in used]
    table = table.clone()
    table[1, 1] = cache.pages
    to_table = torch.tensor([[free[0], -1], [free[1], free[2]]], dtype=torch.int32)
    tokens = torch.tensor([-1, 5, 47, 48, 1 << 30] + [2] * 12 + list(range(0, 40)), dtype=torch.int32)
    start = torch.tensor([0, 17, 57], dtype=torch.int32)
    k = cache.k.cpu().clone()
    A.gather(cache, tokens.to(DEV), start.to(DEV), table.to(DEV), to_table.to(DEV))
    want = k.clone()
    for b in range(2):
        for i, t in enumerate(tokens[start[b]:start[b + 1]].tolist()):
            if t < 0 or t // 16 >= table.shape[1] or i // 16 >= 2:
                continue
            f, to = int(table[b, t // 16]), int(to_table[b, i // 16])
            if 0 <= f < cache.pages and 0 <= to < cache.pages:
                want[to, :, i % 16] = k[f, :, t % 16]
    assert torch.equal(want.view(torch.int16), cache.k.cpu().view(torch.int16))


def test_gather_of_many_sequences_and_heads():
    """More workgroups than a launch holds: the first sequences' tokens, some between and the last one's."""
    from paper_2605_10793_amd import attention as A
    heads, n = 512, 65535
    cache = A.KVCache.empty(8, heads, 16, 64, 16, DEV)
    cache.k.copy_(torch.arange(cache.k.numel(), dtype=torch.int32, device=DEV).view(torch.int16)[:cache.k.numel()].view(cache.k.shape).view(torch.bfloat16))
    cache.v.copy_(cache.k.flip(0).reshape(cache.v.shape))
    counts = torch.zeros(n, dtype=torch.int32)
    table, to_table = torch.full((n, 1), -1, dtype=torch.int32), torch.full((n, 1), -1, dtype=torch.int32)
    for b, to in ((0, 1), (32764, 2), (32768, 3), (n - 1, 4)):
        counts[b], table[b], to_table[b] = 3, 0, to
    tokens = torch.tensor([9, 2, 11] * 4, dtype=torch.int32)
    start = torch.cat([torch.zeros(1, dtype=torch.int32), counts.cumsum(0).to(torch.int32)])
    k, v = (x.view(torch.int16).clone() for x in (cache.k, cache.v))
    A.gather(cache, tokens.to(DEV), start.to(DEV), table.to(DEV), to_table.to(DEV))
    for to in (1, 2, 3, 4):
        k[to, :, :3] = k[0][:, [9, 2, 11]]
        v[to, :, :, :3] = v[0][:, :, [9, 2, 11]]
    assert torch.equal(k, cache.k.view(torch.int16)) and torch.equal(v, cache.v.view(torch.int16))


@pytest.mark.parametrize("bits, page, width", [(8, 16, 64), (8, 64, 128), (4, 16, 128), (4, 32, 64), (4, 256, 128), (16, 32, 128)])
def test_gather_of_tokens_close_to_each_other(bits, page, width):
    """Fours within 16 tokens of a page, at its ends, in any order, one token over and over, fours that are not, and the pool's very last tokens."""
    from paper_2605_10793_amd import attention as A
    g = torch.Generator().manual_seed(bits + page)
    cache = A.KVCache.empty(6, 2, page, width, bits, DEV)
    for x in (cache.k, cache.v, cache.k_scale, cache.v_scale):
        if x is not None:
            x.copy_(torch.randint(0, 255, x.shape, generator=g).to(x.dtype))
    last = page - 1
    picks = [last, last, last, last, last - 3, last, last - 1, last - 2, last - 15, last, last - 7, last - 8, 0, 15, 3, 8, 5, 1, 1, 2, page, last, page + 1, page - 2]
    picks += sorted(torch.randperm(2 * page, generator=g)[:page].tolist()) + torch.randint(0, 2 * page, (page,), generator=g).tolist()
    tokens = torch.tensor(picks[:4 * page], dtype=torch.int32)
    table, to_table = torch.tensor([[3, 5]], dtype=torch.int32), torch.tensor([[0, 4, 2, 1]], dtype=torch.int32)
    start = torch.tensor([0, tokens.shape[0]], dtype=torch.int32)
    want = [None if x is None else x.cpu().clone() for x in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    for i, t in enumerate(tokens.tolist()):
        f, to = int(table[0, t // page]), int(to_table[0, i // page])
        for side, x in enumerate(want):
            if x is not None and side == 1:
                x[to, :, :, i % page] = x[f, :, :, t % page]
            elif x is not None:
                x[to, :, i % page] = x[f, :, t % page]
    A.gather(cache, tokens.to(DEV), start.to(DEV), table.to(DEV), to_table.to(DEV))
    for x, y in zip(want, (cache.k, cache.v, cache.k_scale, cache.v_scale)):
        if x is not None:
            assert torch.equal(x.view(torch.uint8), y.cpu().view(torch.uint8))


@pytest.mark.parametrize("bits, page, width", FORMATS)
@pytest.mark.parametrize("kind, window, cap, biased", [("causal", 0, 0.0, False), ("causal", 1200, 0.0, True), ("holes", 0, 30.0, False)])
def test_few_over_longer_contexts(bits, page, width, kind, window, cap, biased):
    """Contexts that are cut into runs, whatever the format, next to short ones."""
    check(bits, page, width, [2500, 70, 1300], [1, 3, 2], 4, 2, kind=kind, window=window, cap=cap, biased=biased, seed=bits + width, closer=True)
