"""Long pieces of one sequence, every block of which decides some result: one that is lost, taken twice or taken although it is hidden moves the rows
that look at it by a sixteenth of their results or more, sixteen times the bound (that of test_gpu_attention.py: 1.25 * 2^-8 of what is summed).

Each block of 64 tokens has keys that point one of 32 ways and values of its own, signs that differ from block to block; a row of queries looks one way,
so that its result is the mean of the values of some 20 blocks."""
import math

import numpy as np
import pytest

from test_gpu_attention import A, attend64, i32, plan_pages, randn, signed, within  # noqa: F401

pytestmark = pytest.mark.gpu

WAYS, BLOCK = 32, 64
MISSING = {64: [3, 200, 255, 256, 257, 300, 511, 512, 624], 16: [5, 4 * 255 + 1, 4 * 256, 4 * 512 + 3, 2000], 256: [0, 63, 64, 128, 150]}


def blocks_of(tokens, width):
    """Keys and values, [tokens, 1, width]."""
    import torch
    rng = np.random.default_rng(5)
    blocks = -(-tokens // BLOCK)
    key, value = np.zeros((blocks, width), np.float32), rng.choice([-1.0, 1.0], (blocks, width)).astype(np.float32)
    key[np.arange(blocks), (np.arange(blocks) * 7 + np.arange(blocks) // WAYS) % WAYS] = 16.0
    key[:, -1] = -1.0                              # (a zero within the codes, as most keys have one)
    keys = torch.from_numpy(key).cuda().repeat_interleave(BLOCK, 0)[:tokens] + 0.05 * randn(1, tokens, width, dtype="f32")
    values = torch.from_numpy(value).cuda().repeat_interleave(BLOCK, 0)[:tokens] * (1 + 0.2 * randn(2, tokens, width, dtype="f32"))
    return keys[:, None].bfloat16(), values[:, None].bfloat16()


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("width,page", [(64, 64), (128, 64), (64, 16), (128, 256)])
@pytest.mark.parametrize("group,count", [(16, 1), (8, 3), (16, 4)])
@pytest.mark.parametrize("alone", [True, False])
def test_every_block_of_a_long_sequence_counts(A, bits, width, page, group, count, alone):
    """alone: among more sequences than are searched, so that one workgroup takes all of it, run after run of 16384 tokens."""
    import torch
    prefix = 40000 + 17
    others = 530 if alone else 2
    k, v = blocks_of(prefix + count, width)
    table, pages = plan_pages([prefix + count], page, 2, spare=0)
    held, cache = table.copy(), A.KVCache.empty(pages, 1, page, width, bits)
    A.append(cache, k, v, i32([0, prefix + count]), i32([0]), i32(held))
    table[0, MISSING[page]] = -1
    all_tables = np.full((others, table.shape[1]), -1, np.int32)
    all_tables[others // 2] = table[0]
    start = [0] * (others // 2 + 1) + [count] * (others - others // 2)
    prefixes = [0] * others
    prefixes[others // 2] = prefix
    masks = [1 << i for i in range(count)]
    q = torch.zeros(count, group, width, device="cuda:0")
    rows = torch.arange(count * group, device="cuda:0")
    for turn in range(0, WAYS, min(WAYS, count * group)):
        q.zero_()
        q.view(-1, width)[rows, (rows + turn) % WAYS] = 14.0 / 16
        x = q.bfloat16()
        want, size = attend64(x, cache, [0, count], [prefix], table, masks, 1.0)
        got = A.tree_attention(x, cache, i32(start), i32(prefixes), i32(all_tables), mask=signed(masks), max_query=count, max_context=prefix + count, scale=1.0)
        within(got, want, size)
        # the rows' weight lies on their blocks, and each counts
        assert float(want.abs().mean()) > 0.1


def test_the_bound_would_not_pass_one_block_lost_or_taken_twice(A):
    """On the reference alone: what each block of a row's way moves, against the bound."""
    import torch
    tokens, width = 40017, 64
    k, v = (x[:, 0].double() for x in blocks_of(tokens, width))
    for way in range(WAYS):
        w = torch.exp(k[:, way] * 14.0 / 16 - 14)
        w[(torch.arange(tokens, device="cuda:0") // BLOCK % 97) == 3] = 0          # (some not seen)
        parts = torch.stack([(torch.nn.functional.pad(w, (0, -tokens % BLOCK)).view(-1, BLOCK)).sum(1)], 1)
        sums = torch.nn.functional.pad(w[:, None] * v, (0, 0, 0, -tokens % BLOCK)).view(-1, BLOCK, width).sum(1)
        o = sums.sum(0) / parts.sum()
        bound = 2.25 * 2.0 ** -8 * (w[:, None] * v.abs()).sum(0) / parts.sum()
        heavy = parts[:, 0] > 0.02 * parts.sum()
        assert heavy.sum() >= 16 and float(parts[heavy].sum() / parts.sum()) > 0.9
        for times in (-1.0, 1.0):
            moved = ((sums.sum(0) + times * sums) / (parts.sum() + times * parts) - o).abs() / bound
            assert float(moved.amax(1)[heavy].min()) > 2
