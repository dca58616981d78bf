"""Tree attention over caches as others may have filled them, over every way the work is cut, and the layer that runs the attention operators
together.  References and bounds are those of test_gpu_attention.py:

  results   v |o| + 1.25 v sum p |value| + 4 u (sum p of the 256 steps and the offset that a value is made of); u = 2^-24, v = 2^-8.
            Keys are held to offsets and steps whose 32-bit rounding moves a score by less than 2^-10: 2^-22 scale sum |q| (256 step + |offset|)
            with |q| some 100 a row, scale 0.09, and 10 for the bracket, is 2e-5.  Values of any pair: the bound's last term follows the pair.
  equal     whatever is decided without rounding, or by the same operations on the same numbers
"""
import numpy as np
import pytest

from test_gpu_attention import A, attend64, filled_cache, i32, plan_pages, randn, signed, tree_masks, within  # noqa: F401

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ every cut of the rows

ROWS = [  # group, counts: rows a cache head = group * count, one of them of another size
    (5, [8, 3]), (8, [9, 9]), (4, [33, 1]), (8, [24, 2]), (3, [64, 64]), (8, [64, 17]), (64, [4, 1]), (2, [16, 8]), (1, [20, 20]),
]


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("width,page", [(64, 16), (64, 128), (128, 32), (128, 64)])
@pytest.mark.parametrize("rows", ROWS, ids=str)
def test_row_tiles(A, rows, width, page, bits):
    group, counts = rows
    prefix = [700, 333]
    cache, table = filled_cache(A, [p + n for p, n in zip(prefix, counts)], page, 1, width, bits, 31)
    start = [0, counts[0], sum(counts)]
    q = randn(7, sum(counts), group, width)
    masks = [m for b, n in enumerate(counts) for m in tree_masks(n, b)]
    want, size = attend64(q, cache, start, prefix, table, masks, width ** -0.5)
    for context in (None, max(p + n for p, n in zip(prefix, counts))):
        got = A.tree_attention(q, cache, i32(start), i32(prefix), i32(table), mask=signed(masks), max_query=max(counts), max_context=context)
        within(got, want, size)


# ------------------------------------------------------------------------------------------------ codes and pairs of any making

def pair_kinds(cache, which, seed):
    """Every token's pair one of: as the quantiser makes them; a zero far outside the codes, on either side; a negative step; a constant
    (step 0, whatever the codes); a step below what a quotient by it can hold; all zero."""
    import torch
    scale = cache.k_scale if which == "k" else cache.v_scale
    codes = cache.k if which == "k" else cache.v
    g = torch.Generator(device="cuda:0")
    g.manual_seed(seed)
    codes.copy_(torch.randint(0, 256, codes.shape, generator=g, device="cuda:0"))
    top = 255.0 if cache.bits == 8 else 15.0
    n = scale[..., 0].numel()
    step = (0.5 + torch.rand(n, generator=g, device="cuda:0")) * 2 / top
    zero = torch.rand(n, generator=g, device="cuda:0") * top
    kind = torch.randint(0, 12, (n,), generator=g, device="cuda:0")
    offset = -step * zero
    offset = torch.where(kind == 1, 1.5 + zero / top, offset)
    offset = torch.where(kind == 2, -5.0 - zero / top, offset)
    step = torch.where(kind == 3, -step, step)
    offset = torch.where(kind == 3, -offset, offset)
    step = torch.where(kind == 4, torch.zeros_like(step), step)
    step = torch.where(kind == 5, torch.full_like(step, 1e-35), step)
    step = torch.where(kind == 6, torch.full_like(step, 1e-41), step)
    step = torch.where(kind == 7, torch.zeros_like(step), step)
    offset = torch.where(kind == 7, torch.zeros_like(step), offset)
    scale.copy_(torch.stack([step, offset], -1).view(scale.shape))


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("group,count", [(4, 1), (5, 5), (8, 12), (6, 40)])
def test_any_pair_is_step_times_code_plus_offset(A, bits, page, group, count):
    width, prefix = 128, [900, 65]
    cache, table = filled_cache(A, [p + count for p in prefix], page, 1, width, bits, 3)
    pair_kinds(cache, "k", 1)
    pair_kinds(cache, "v", 2)
    start = [0, count, 2 * count]
    q = randn(4, 2 * count, group, width)
    masks = tree_masks(count, 0) + tree_masks(count, 1)
    want, size = attend64(q, cache, start, prefix, table, masks, width ** -0.5)
    got = A.tree_attention(q, cache, i32(start), i32(prefix), i32(table), mask=signed(masks), max_query=count)
    within(got, want, size)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("group,count", [(2, 1), (8, 12)])
def test_constant_rows(A, bits, group, count):
    """Keys and values constant over the width, as `append` quantises them: step 0, and the value as it is."""
    import torch
    lengths, width = [300 + count], 64
    table, pages = plan_pages(lengths, 32, 5)
    cache = A.KVCache.empty(pages, 1, 32, width, bits)
    k, v = randn(1, lengths[0], 1, 1).expand(-1, 1, width).contiguous(), randn(2, lengths[0], 1, 1).expand(-1, 1, width).contiguous()
    A.append(cache, k, v, i32([0, lengths[0]]), i32([0]), i32(table))
    q = randn(3, count, group, width)
    want, size = attend64(q, cache, [0, count], [300], table, None, width ** -0.5)
    got = A.tree_attention(q, cache, i32([0, count]), i32([300]), i32(table), max_query=count)
    within(got, want, size)
    assert torch.equal(got, got[..., :1].expand_as(got))


# ------------------------------------------------------------------------------------------------ pages that do not exist

@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("group,count", [(4, 1), (8, 3), (6, 30)])
def test_holes(A, bits, page, group, count):
    """Tokens without a page anywhere, at the ends, a whole sequence of them: not seen, whatever lies in page 0."""
    import torch
    prefix = [2000, 40, 1500]
    cache, table = filled_cache(A, [p + count for p in prefix], page, 2, 64, bits, 6)
    rng = np.random.default_rng(page)
    holes = table.copy()
    holes[0, rng.random(holes.shape[1]) < 0.4] = -1
    holes[1, :] = np.array([1 << 30, -5])[rng.integers(0, 2, holes.shape[1])]
    holes[2, 0], holes[2, (1500 + count - 1) // page] = cache.pages, -(1 << 31)
    start = [0, count, 2 * count, 3 * count]
    q = randn(8, 3 * count, 2 * group, 64)
    want, size = attend64(q, cache, start, prefix, holes, None, 0.125)
    got = A.tree_attention(q, cache, i32(start), i32(prefix), i32(holes), max_query=count)
    within(got, want, size)
    assert torch.all(got[count:2 * count] == 0)


# ------------------------------------------------------------------------------------------------ many sequences, long pieces

@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("count,group", [(2, 2), (5, 8)])
def test_more_sequences_than_are_searched(A, bits, count, group):
    """Beyond 512 sequences each has a workgroup; one of them is longer than the run after which put-off blocks are made up for."""
    import torch
    sequences, width, page = 530, 64, 64
    rng = np.random.default_rng(1)
    counts = rng.integers(0, count + 1, sequences)
    prefix = rng.integers(0, 90, sequences)
    counts[77], prefix[77] = count, 40000
    cache, table = filled_cache(A, [int(p + n) for p, n in zip(prefix, counts)], page, 1, width, bits, 2)
    table[77, [3, 200, 259, 300, 624]] = -1
    start = [0] + [int(x) for x in np.cumsum(counts)]
    q = randn(9, start[-1], group, width)
    got = A.tree_attention(q, cache, i32(start), i32(prefix), i32(table), max_query=count)
    want, size = attend64(q, cache, start, [int(p) for p in prefix], table, None, 0.125)
    within(got, want, size)
    few = A.tree_attention(q[start[70]:start[80]], cache, i32([s - start[70] for s in start[70:81]]), i32(prefix[70:80]), i32(table[70:80]), max_query=count)
    within(few, want[start[70]:start[80]], size[start[70]:start[80]])


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("count,group", [(1, 1), (1, 20), (40, 1)])
def test_runs_over_many_sequences(A, bits, count, group):
    """So many heads that a workgroup's run spans several sequences, empty ones among them, and one sequence several runs."""
    import torch
    heads, width, page = 32 if group == 1 else 16, 64, 32
    prefix = [70, 0, 0, 3000, 5, 64, 0, 1, 130, 63, 0, 0, 900, 10, 40]
    counts = [count, 0, count, count, 1, 0, 0, 1, count, 1, 0, 0, 1, 0, 1]
    cache, table = filled_cache(A, [p + n for p, n in zip(prefix, counts)], page, heads, width, bits, 13)
    start = [0] + [int(x) for x in np.cumsum(counts)]
    q = randn(14, start[-1], heads * group, width)
    want, size = attend64(q, cache, start, prefix, table, None, 0.125)
    got = A.tree_attention(q, cache, i32(start), i32(prefix), i32(table), max_query=count)
    within(got, want, size)
    assert torch.equal(got, A.tree_attention(q, cache, i32(start), i32(prefix), i32(table), max_query=count))


@pytest.mark.parametrize("sequences", [1, 64, 65, 4097])
def test_append_finds_every_sequence(A, sequences):
    import torch
    rng = np.random.default_rng(sequences)
    counts, prefix = rng.integers(0, 4, sequences), rng.integers(0, 60, sequences)
    counts[-1], counts[sequences // 2] = 2, 70
    start = np.concatenate([[0], np.cumsum(counts)])
    width, page, columns = 64, 32, 5
    table = np.arange(sequences * columns, dtype=np.int32).reshape(sequences, columns)
    cache = A.KVCache.empty(sequences * columns, 1, page, width)
    cache.k.fill_(7.0)
    cache.v.fill_(7.0)
    k, v = randn(1, start[-1], 1, width), randn(2, start[-1], 1, width)
    A.append(cache, k, v, i32(start), i32(prefix), i32(table))
    at = np.concatenate([b * columns * page + prefix[b] + np.arange(counts[b]) for b in range(sequences)])
    at = torch.from_numpy(at).cuda()
    want = torch.full((sequences * columns * page, width), 7.0, dtype=torch.bfloat16, device="cuda:0")
    want[at] = k[:, 0]
    assert torch.equal(cache.k.view(-1, width), want)
    want.fill_(7.0)
    want[at] = v[:, 0]
    assert torch.equal(cache.v.transpose(2, 3).reshape(-1, width), want)


# ------------------------------------------------------------------------------------------------ the operators together

@pytest.mark.parametrize("bits", [16, 8, 4])
def test_the_layer_serves_calibrates_and_learns(A, bits):
    """Prompts in chunks, then drafted trees of which a path stays: the cache holds what the same tokens leave there as a chain, every output
    is the attention over it, the calibrator has seen the committed rows, and the gradients are the operator's."""
    import torch
    from paper_2605_10793_amd import binding
    from paper_2605_10793_amd.layer import AttentionLayer
    heads, kv, width, page, B = 8, 2, 128, 32, 3
    plan = A.Rotary(width)
    wq, wk = 1 + randn(1, width) / 4, 1 + randn(2, width) / 4
    lengths = [150, 90, 201]
    draft, keep = [5, 0, 7], [[0, 2], [], [0, 1, 4]]
    masks = [tree_masks(n, 3) for n in draft]
    masks[0][2], masks[2][1], masks[2][4] = 0b101, 0b11, 0b10011
    table, pages = plan_pages([n + 8 for n in lengths], page, 1)
    prompts = [randn(10 + b, n, heads + 2 * kv, width) for b, n in enumerate(lengths)]
    drafts = [randn(20 + b, n, heads + 2 * kv, width) for b, n in enumerate(draft)]

    def offsets(counts):
        return i32(np.concatenate([[0], np.cumsum(counts)]))

    def feed(layer, rows):
        at = [0] * B
        while any(a < len(r) for a, r in zip(at, rows)):
            n = [min(50, len(r) - a) for a, r in zip(at, rows)]
            out = layer.step(torch.cat([r[a:a + m] for a, m, r in zip(at, n, rows)]), offsets(n))
            layer.commit(offsets(n))
            at = [a + m for a, m in zip(at, n)]
        return out

    R0 = torch.linalg.qr(torch.randn(heads, width, width, generator=torch.Generator().manual_seed(1)))[0].numpy()
    cals = [binding.Calibrator(heads * width, heads, "bf16", R0, max_tokens=512) for _ in range(2)]
    try:
        layers, caches = [], []
        for cal in cals:
            cache = A.KVCache.empty(pages, kv, page, width, bits)
            for x in (cache.k, cache.v, cache.k_scale, cache.v_scale):
                if x is not None:
                    x.zero_()
            caches.append(cache)
            layers.append(AttentionLayer(plan, wq, wk, cache, i32(table), calibrator=cal))
        feed(layers[0], prompts)
        depth = torch.tensor([bin(m).count("1") - 1 for ms in masks for m in ms], device="cuda:0")
        fused = torch.cat(drafts)
        out = layers[0].step(fused, offsets(draft), depth, signed([m for ms in masks for m in ms]), max_query=7)
        first = np.concatenate([[0], np.cumsum(draft)])

        # the outputs, from the drafted cache
        pos = torch.cat([lengths[b] + depth[first[b]:first[b + 1]] for b in range(B)])
        q = A.qk_norm_rotary(plan, fused[:, :heads], fused[:, heads:heads + kv], wq, wk, pos, eps=1e-6)[0]
        want, size = attend64(q, caches[0], first, lengths, table, [m for ms in masks for m in ms], width ** -0.5)
        within(out, want, size)

        q_grad, k_grad = randn(30, *fused[:, :heads].shape), randn(31, *fused[:, heads:heads + kv].shape)
        for x, y in zip(layers[0].gradients(q_grad, k_grad),
                        A.qk_norm_rotary_backward(plan, fused[:, :heads], fused[:, heads:heads + kv], wq, wk, pos, q_grad, k_grad)):
            assert torch.equal(x, y)

        rows = [int(first[b]) + i for b in range(B) for i in keep[b]]
        layers[0].commit(offsets([len(x) for x in keep]), torch.tensor(rows, device="cuda:0"))
        feed(layers[1], [torch.cat([p, d[x]]) for p, d, x in zip(prompts, drafts, keep)])
        assert torch.equal(layers[0].prefix, layers[1].prefix)
        done = layers[1].prefix.tolist()
        for b in range(B):
            for t in range(done[b]):
                p, s = int(table[b, t // page]), t % page
                assert torch.equal(caches[0].k[p, :, s], caches[1].k[p, :, s]) and torch.equal(caches[0].v[p, :, :, s], caches[1].v[p, :, :, s])
                if bits != 16:
                    assert torch.equal(caches[0].k_scale[p, :, s], caches[1].k_scale[p, :, s])
        assert [s["rows"] for s in cals[0].batch_stats()] == [sum(done)] * heads
        cals[0].update_rotation()
    finally:
        for cal in cals:
            cal.close()
