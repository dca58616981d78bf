"""Weights of attention over codes: a token's weight counts alike in the result and in the sum that divides it, however it was rounded.

Where one token has all the weight, the result is that token's value: its step times its code plus its offset.  What the arithmetic may add to the
rounding of the result (half a unit of bf16, 2^-8 of the power of two below it) is
  2^-22 (256 step + |offset|)   the sums of code and offset apart in 32 bits, four units of their terms
  2^-20 |value|                 quotient and factors in 32 bits; all other tokens' weights together, e^-40 of the first
"""
import numpy as np
import pytest

from test_gpu_attention import A, filled_cache, i32, randn, signed, values_of  # noqa: F401

pytestmark = pytest.mark.gpu


def to_bf16_of(got, want, terms):
    """got is bf16, want the value in 64 bits."""
    import torch
    half = torch.exp2(torch.floor(torch.log2(want.abs().clamp(min=1e-30))) - 8)
    return float(((got.double() - want).abs() / (half + 2.0 ** -20 * want.abs() + 2.0 ** -22 * terms)).max())


def rows_of(kind, seed, tokens, heads, width):
    """Values whose zero lies among their codes, above them or below them; 8-bit steps as wide as a unit of bf16, so that values lie between its numbers."""
    import torch
    x = randn(seed, tokens, heads, width, dtype="f32")
    size = 1 + torch.rand(tokens, 1, 1, generator=torch.Generator(device="cuda:0").manual_seed(seed), device="cuda:0")
    if kind != "among":
        x = size + 2 * torch.rand(tokens, heads, width, generator=torch.Generator(device="cuda:0").manual_seed(seed + 1), device="cuda:0")
        x = -x if kind == "above" else x
    return x.to(torch.bfloat16)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("kind", ["among", "above", "below"])
@pytest.mark.parametrize("width,page", [(128, 64), (64, 16)])
@pytest.mark.parametrize("group,count", [(4, 1), (8, 3), (8, 8), (4, 40)])
def test_one_token_with_all_the_weight(A, bits, kind, width, page, group, count):
    """A committed token that outweighs all others, at places in blocks of every kind; then new tokens that see themselves alone."""
    import torch
    heads, prefix = 2, 333
    cache, table = filled_cache(A, [prefix + count], page, heads, width, bits, 1)
    k = 0.1 * randn(2, prefix + count, heads, width, dtype="f32")
    v = rows_of(kind, 3, prefix + count, heads, width)
    start, lengths, tab = i32([0, count]), i32([prefix]), i32(table)
    q = (1 + 0.2 * randn(4, count, heads * group, width, dtype="f32").abs()).to(torch.bfloat16)
    for at in (0, 70, 200, 255, 319, 320, prefix - 1):
        one = k.clone()
        one[at] = torch.linspace(0.9, 1.0, width, device="cuda:0")
        A.append(cache, one.to(torch.bfloat16), v, i32([0, prefix + count]), i32([0]), tab)
        got = A.tree_attention(q, cache, start, lengths, tab, max_query=count, max_context=prefix + count, scale=2.0)
        value, terms = values_of(cache, "v", table[0], prefix + count)
        want = value[:, at].repeat_interleave(group, 0).expand_as(got)
        assert to_bf16_of(got, want, terms[:, at].repeat_interleave(group, 0)[None, :, None]) <= 1, at
    # (nothing committed: the same tokens as new ones)
    A.append(cache, k[:count].to(torch.bfloat16), v[:count], start, i32([0]), tab)
    got = A.tree_attention(q, cache, start, i32([0]), tab, mask=signed([1 << i for i in range(count)]), max_query=count)
    value, terms = values_of(cache, "v", table[0], count)
    want, terms = (x.transpose(0, 1).repeat_interleave(group, 1) for x in (value, terms[..., None]))
    assert to_bf16_of(got, want, terms) <= 1


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("kind", ["among", "above", "below"])
@pytest.mark.parametrize("group,count", [(4, 1), (8, 3), (8, 8), (4, 40)])
def test_tokens_of_one_value(A, bits, kind, group, count):
    """All tokens of a head hold the same value, and any weights give it."""
    import torch
    heads, width, prefix = 2, 128, 1000
    cache, table = filled_cache(A, [prefix + count], 64, heads, width, bits, 1)
    k, v = randn(2, prefix + count, heads, width), rows_of(kind, 3, 1, heads, width).expand(prefix + count, -1, -1)
    A.append(cache, k, v, i32([0, prefix + count]), i32([0]), i32(table))
    q = randn(4, count, heads * group, width)
    got = A.tree_attention(q, cache, i32([0, count]), i32([prefix]), i32(table), max_query=count, max_context=prefix + count, scale=0.3)
    value, terms = values_of(cache, "v", table[0], 1)
    want, terms = (x[:, 0].repeat_interleave(group, 0)[None].expand(count, -1, -1) for x in (value, terms[..., None]))
    # (a lane adds up to 64 terms in series, and half as many products' sums, each to 2^-24 of what it has: 2^-17 of the terms)
    assert to_bf16_of(got, want, 32 * terms) <= 1


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("kind", ["among", "above", "below"])
@pytest.mark.parametrize("group,count", [(8, 1), (8, 3), (8, 8), (4, 40)])
def test_errors_are_those_of_two_roundings(A, bits, kind, group, count):
    """The squares of all errors together: the result's rounding, a unit^2 / 12 each, and the weights', up to 2^-14 / 12 of their squares, which the
    sum that divides takes part in, so that they count by the distance of their values from the result.  A tenth more for some ten thousand draws."""
    import torch
    heads, width, prefix, scale = 8, 128, 640, 0.25
    cache, table = filled_cache(A, [prefix + count], 64, heads, width, bits, 1)
    k, v = randn(2, prefix + count, heads, width), rows_of(kind, 3, prefix + count, heads, width)
    A.append(cache, k, v, i32([0, prefix + count]), i32([0]), i32(table))
    square = limit = spread = 0.0
    for seed in range(4):
        q = randn(10 + seed, count, heads * group, width)
        got = A.tree_attention(q, cache, i32([0, count]), i32([prefix]), i32(table), max_query=count, max_context=prefix + count, scale=scale)
        keys, values = values_of(cache, "k", table[0], prefix + count)[0], values_of(cache, "v", table[0], prefix + count)[0]
        for h in range(heads):
            s = q[:, h * group:(h + 1) * group].double() @ keys[h].t().contiguous() * scale
            hidden = torch.arange(prefix + count, device="cuda:0") > prefix + torch.arange(count, device="cuda:0")[:, None, None]
            p = torch.softmax(s.masked_fill(hidden, -float("inf")), -1)
            want = p @ values[h]
            unit = torch.exp2(torch.floor(torch.log2(want.abs().clamp(min=1e-30))) - 7)
            away = (p.square() @ values[h].square() - 2 * want * (p.square() @ values[h]) + want.square() * p.square().sum(-1, keepdim=True)).sum()
            square += float((got[:, h * group:(h + 1) * group].double() - want).square().sum())
            limit += float(unit.square().sum()) / 12 + float(away) * 2.0 ** -14 / 12
            spread += float(p.square().sum(-1).mean()) / (4 * heads)
    assert spread > 0.1            # few tokens count, or the weights' rounding would not
    assert square <= 1.1 * limit, square / limit
