"""The attention layer's operators (paper_2605_10793_amd.attention) against plain implementations in 64 bits.

Tolerances, from the arithmetic (u = 2^-24 for fp32, v = 2^-8 the rounding to bf16, whose
significand has 8 bits):
  rotary      the angle is rounded to 32 bits as a fraction of a turn (2^-25 turns, 2e-7 in the angle), sine and cosine to some
              2 u, products and their sum to 3 u: below 1e-6 (|a| + |b|) m, and v |y| where the result is bf16
  norm        the row's sum is a tree of 32-bit sums and its root and quotient are rounded: below 8 u relative on top of that
  gradient    a product of five such factors and a sum over the width: below 2e-6 times the sum of the terms' magnitudes
  weights     sums of n terms in a tree at most 64 long in series: below 64 u times the sum of the terms' magnitudes
  append      codes, steps and offsets are decided by single 32-bit operations: equal; values: one rounding to bf16
  attention   v |o| for the result and v for each weight, i.e. v sum p |v| / sum p, a quarter of it more for scores and sums in 32 bits;
              with codes the sums' terms are not the values but code and offset apart, up to 256 steps and the offset: 4 u of those
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

V = 2.0 ** -8


@pytest.fixture(scope="module")
def A():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device")
    from paper_2605_10793_amd import attention
    return attention


def gen(seed):
    import torch
    g = torch.Generator(device="cuda:0")
    g.manual_seed(seed)
    return g


def randn(seed, *shape, dtype="bf16"):
    import torch
    x = torch.randn(*shape, device="cuda:0", generator=gen(seed))
    return x.to(torch.bfloat16 if dtype == "bf16" else torch.float32)


# ------------------------------------------------------------------------------------------------ rotary positions and norms

def pairs(x, part, interleaved):
    return (x[..., 0:part:2], x[..., 1:part:2]) if interleaved else (x[..., :part // 2], x[..., part // 2:part])


def rotate64(x, positions, turns, part, interleaved, magnitude, transposed=False):
    """The definition on float64 rows [tokens, heads, width]; also the sum of the magnitudes of every result's terms."""
    import torch
    t = positions.double()[:, None] * turns
    t = 2 * math.pi * (t - torch.floor(t))
    cos, sin = torch.cos(t)[:, None], torch.sin(t)[:, None]
    if transposed:
        sin = -sin
    a, b = pairs(x, part, interleaved)
    y, size = x.clone(), x.abs().clone()
    ya, yb = pairs(y, part, interleaved)
    sa, sb = pairs(size, part, interleaved)
    ya.copy_((a * cos - b * sin) * magnitude)
    yb.copy_((b * cos + a * sin) * magnitude)
    sa.copy_((a.abs() + b.abs()) * magnitude)
    sb.copy_((a.abs() + b.abs()) * magnitude)
    return y, size


def within(got, want, bound, dtype="bf16"):
    err = (got.double() - want).abs()
    limit = bound + (V * want.abs() if dtype == "bf16" else 0) + 1e-38
    worst = float((err / limit).max()) if err.numel() else 0.0
    assert worst <= 1.0, worst


ROTARY = [  # tokens, q heads, k heads, width, part, interleaved, scaling
    (1, 32, 8, 128, 128, False, "none"), (1, 1, 0, 64, 64, True, "linear"), (3, 5, 1, 128, 64, True, "bands"), (17, 32, 8, 96, 48, False, "ramp"),
    (129, 7, 7, 80, 80, False, "base"), (64, 3, 2, 80, 40, True, "none"), (33, 2, 1, 256, 256, False, "bands"), (5, 1, 1, 512, 512, True, "none"),
    (9, 4, 2, 6, 2, False, "none"), (2500, 8, 2, 64, 62, False, "ramp"), (4500, 6, 2, 128, 128, True, "linear"), (11, 1, 3, 510, 254, False, "none"),
]
FACTORS = {"none": {}, "linear": dict(factor=4.0), "base": dict(factor=2.5), "bands": dict(factor=8.0, low=1.0, high=4.0, context=8192.0),
           "ramp": dict(factor=16.0, low=1.0, high=32.0, context=4096.0)}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", ROTARY, ids=str)
def test_rotary_and_its_transpose(A, case, dtype):
    import torch
    T, hq, hk, width, part, inter, scaling = case
    plan = A.Rotary(part, 10000.0, interleaved=inter, scaling=scaling, **FACTORS[scaling])
    fused = randn(T + width, T, hq + hk, width, dtype=dtype)
    q, k = fused[:, :hq], fused[:, hq:] if hk else None
    pos = torch.randint(0, 1 << 20, (T,), generator=gen(5), device="cuda:0")
    for transposed in (False, True):
        got = A.rotary(plan, q, pos, k=k, transposed=transposed)
        for x, y in zip((q, k), got if hk else (got,)):
            want, size = rotate64(x.double(), pos, plan.turns, part, inter, plan.magnitude, transposed)
            within(y, want, 1e-6 * size, dtype)
            assert torch.equal(y[..., part:], x[..., part:])


def test_rotary_frequencies_follow_their_definitions(A):
    def want(part, theta, scaling, factor=1.0, low=0.0, high=0.0, context=0.0):
        out = []
        for j in range(part // 2):
            f = (theta * factor ** (part / (part - 2)) if scaling == "base" else theta) ** (-2 * j / part)
            turns = context * f / (2 * math.pi)
            if scaling == "linear":
                f /= factor
            if scaling == "bands":
                keep = min(1.0, max(0.0, (turns - low) / (high - low)))
                f = f * keep + f / factor * (1 - keep)
            if scaling == "ramp":
                at = [part * math.log(context / (r * 2 * math.pi)) / (2 * math.log(theta)) for r in (high, low)]
                a, b = max(math.floor(at[0]), 0), min(math.ceil(at[1]), part - 1)
                keep = 1 - min(1.0, max(0.0, (j - a) / max(b - a, 1e-3)))
                f = f * keep + f / factor * (1 - keep)
            out.append(f / (2 * math.pi))
        return np.array(out)

    for part in (2, 40, 64, 128, 512):
        for scaling, more in FACTORS.items():
            if scaling == "base" and part == 2:
                continue
            for theta in (10000.0, 500000.0):
                plan = A.Rotary(part, theta, scaling=scaling, **more)
                np.testing.assert_allclose(plan.turns.cpu().numpy(), want(part, theta, scaling, **more), rtol=1e-13)
                assert plan.magnitude == pytest.approx(0.1 * math.log(16.0) + 1 if scaling == "ramp" else 1.0, rel=1e-7)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotary_takes_any_strides_and_writes_nothing_else(A, dtype):
    import torch
    plan = A.Rotary(32, interleaved=False)
    T, heads, width = 21, 3, 48
    pos = torch.arange(T, device="cuda:0") - 7                                 # negative positions too
    base = randn(3, T * 400 + 64, dtype=dtype)
    views = [base[1:].as_strided((T, heads, width), (400, 67, 1)),             # odd strides, odd offset
             base.as_strided((T, heads, width), (width, T * width, 1)),        # heads outermost
             base.as_strided((T, heads, width), (width, 0, 1)),                # one row for all heads
             base.as_strided((T, heads, width), (0, width, 1))]                # one for all tokens
    for x in views:
        want, size = rotate64(x.double(), pos, plan.turns, 32, False, 1.0)
        within(A.rotary(plan, x, pos), want, 1e-6 * size, dtype)
        room = torch.full((T * 500 + 64,), 7.0, device="cuda:0", dtype=x.dtype)
        out = room[3:].as_strided((T, heads, width), (500, 71, 1))
        A.rotary(plan, x, pos, out=out)
        within(out, want, 1e-6 * size, dtype)
        keep = torch.ones_like(room, dtype=torch.bool)
        keep[3:].as_strided((T, heads, width), (500, 71, 1)).fill_(False)
        assert torch.all(room[keep] == 7.0)
    fused = randn(4, T, 2 * heads, width, dtype=dtype)                          # in place, in a slice of a fused tensor
    before = fused.clone()
    A.rotary(plan, fused[:, :heads], pos, out=fused[:, :heads])
    want, size = rotate64(before[:, :heads].double(), pos, plan.turns, 32, False, 1.0)
    within(fused[:, :heads], want, 1e-6 * size, dtype)
    assert torch.equal(fused[:, heads:], before[:, heads:])


def test_rotary_keeps_far_positions_and_special_values(A):
    import torch
    plan = A.Rotary(64, 10000.0)
    pos = torch.tensor([0, 1, 1 << 24, (1 << 31) + 5, 10 ** 9], device="cuda:0")
    x = randn(9, 5, 2, 64, dtype="f32")
    want, size = rotate64(x.double(), pos, plan.turns, 64, False, 1.0)
    within(A.rotary(plan, x, pos), want, 2e-6 * size, "f32")                    # 1e9 turns leave 2^-23 of one in 64 bits
    assert torch.equal(A.rotary(plan, x, pos)[0], x[0])
    x[1, 0, 3], x[1, 1, 40] = math.inf, math.nan
    y = A.rotary(plan, x, pos)
    assert torch.equal(torch.isfinite(y).all(-1), torch.isfinite(x).all(-1))    # no row touches another
    empty = A.rotary(plan, x[:0], pos[:0])
    assert empty.shape == (0, 2, 64)


def norm64(x, w, eps):
    rstd = 1 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    return x * rstd, rstd, x * rstd * w


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", ROTARY, ids=str)
def test_norm_and_rotary_and_their_gradients(A, case, dtype):
    import torch
    T, hq, hk, width, part, inter, scaling = case
    hk = max(hk, 1)
    eps = 1e-5
    plan = A.Rotary(part, 10000.0, interleaved=inter, scaling=scaling, **FACTORS[scaling])
    fused = randn(2 * T + width, T, hq + hk, width, dtype=dtype) * torch.linspace(0.2, 3, width, device="cuda:0").to(torch.bfloat16)
    if T > 2:
        fused[1] = 0                                                            # rows of zeros
    q, k = fused[:, :hq], fused[:, hq:]
    wq, wk = 1 + randn(1, width, dtype=dtype) / 4, 1 + randn(2, width, dtype=dtype) / 4
    pos = torch.randint(0, 1 << 17, (T,), generator=gen(5), device="cuda:0")
    out = A.qk_norm_rotary(plan, q, k, wq, wk, pos, eps)
    gq, gk = randn(7, T, hq, width, dtype=dtype), randn(8, T, hk, width, dtype=dtype)
    back = A.qk_norm_rotary_backward(plan, q, k, wq, wk, pos, gq, gk, eps)
    again = A.qk_norm_rotary_backward(plan, q, k, wq, wk, pos, gq, gk, eps)
    assert all(torch.equal(a, b) for a, b in zip(back, again))                  # sums in a fixed order
    for i, (x, w, g) in enumerate(((q, wq, gq), (k, wk, gk))):
        x, w, g = x.double(), w.double(), g.double()
        unit, rstd, u = norm64(x, w, eps)
        want, size = rotate64(u, pos, plan.turns, part, inter, plan.magnitude)
        within(out[i], want, 2e-6 * size, dtype)
        h, size = rotate64(g, pos, plan.turns, part, inter, plan.magnitude, True)
        mean = (h * w * unit).mean(-1, keepdim=True)
        want = rstd * (h * w - unit * mean)
        terms = rstd * (size * w.abs() + unit.abs() * (size * w.abs() * unit.abs()).mean(-1, keepdim=True))
        within(back[i], want, 2e-6 * terms, dtype)
        dw = back[2 + i]
        assert dw.dtype == torch.float32
        err = (dw.double() - (h * unit).sum((0, 1))).abs()
        assert torch.all(err <= 64 * 2.0 ** -24 * (size * unit.abs()).sum((0, 1)) + 1e-38)


def test_norm_gradients_against_differences(A):
    """The derivative of a weighted sum of the 64-bit results along random directions of inputs and weights."""
    import torch
    T, hq, hk, width, part = 6, 4, 2, 64, 48
    plan = A.Rotary(part, 10000.0, interleaved=True)
    eps = 1e-4
    q, k = randn(1, T, hq, width, dtype="f32"), randn(2, T, hk, width, dtype="f32")
    wq, wk = 1 + randn(3, width, dtype="f32") / 4, 1 + randn(4, width, dtype="f32") / 4
    gq, gk = randn(5, T, hq, width, dtype="f32"), randn(6, T, hk, width, dtype="f32")
    pos = torch.arange(T, device="cuda:0") * 31
    back = A.qk_norm_rotary_backward(plan, q, k, wq, wk, pos, gq, gk, eps)

    def value(args):
        total = 0.0
        for x, w, g in ((args[0], args[2], gq), (args[1], args[3], gk)):
            total = total + (rotate64(norm64(x, w, eps)[2], pos, plan.turns, part, True, 1.0)[0] * g.double()).sum()
        return float(total)

    at = [x.double() for x in (q, k, wq, wk)]
    for i in range(4):
        for seed in range(3):
            way = torch.randn(at[i].shape, generator=gen(20 + seed), device="cuda:0", dtype=torch.float64)
            h = 1e-5
            up, down = [list(at) for _ in range(2)]
            up[i], down[i] = at[i] + h * way, at[i] - h * way
            slope = (value(up) - value(down)) / (2 * h)
            terms = float((back[i].double() * way).abs().sum())
            # 32-bit gradients (2e-6 of their terms) and the difference's own h^2 and 1/h parts (1e-16 * value / h, some 1e-9)
            assert abs(float((back[i].double() * way).sum()) - slope) <= 4e-6 * terms + 1e-6


def test_shared_gradient_rows(A):
    """A gradient that is one row for all heads (strides of 0) is that row's copies' gradient."""
    import torch
    plan = A.Rotary(128)
    q, k = randn(1, 40, 8, 128), randn(2, 40, 2, 128)
    w = 1 + randn(3, 128) / 4
    pos = torch.arange(40, device="cuda:0")
    row, gk = randn(4, 40, 1, 128), randn(5, 40, 2, 128)
    a = A.qk_norm_rotary_backward(plan, q, k, w, w, pos, row.expand(40, 8, 128), gk)
    b = A.qk_norm_rotary_backward(plan, q, k, w, w, pos, row.expand(40, 8, 128).contiguous(), gk)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


# ------------------------------------------------------------------------------------------------ the cache

def quantise32(rows, bits):
    """numpy's single 32-bit operations, in the definition's order."""
    rows = rows.astype(np.float32)
    top = np.float32(2 ** bits - 1)
    lo, hi = rows.min(-1, keepdims=True), rows.max(-1, keepdims=True)
    step = (hi - lo) / top
    safe = np.where(step == 0, np.float32(1), step)
    zeta = -np.rint(lo / safe)
    code = np.where(step == 0, np.float32(0), np.clip(np.rint(rows / safe) + zeta, np.float32(0), top))
    offset = np.where(step == 0, lo, -(step * zeta))
    return code, step, offset


def pack(code, bits):
    code = code.astype(np.uint8)
    half = code.shape[-1] // 2
    return code if bits == 8 else code[..., :half] | code[..., half:] << 4


def i32(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda:0")


def plan_pages(lengths, page, seed, spare=2):
    """Scattered pages for sequences of these lengths: (table, pages of the pool); unused entries name no page."""
    rng = np.random.default_rng(seed)
    need = [(n + page - 1) // page for n in lengths]
    order = rng.permutation(sum(need) + spare)
    table = np.full((len(lengths), max(max(need), 1)), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, sum(need) + spare


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("width,page,heads,counts,prefix", [
    (128, 64, 8, [1] * 5, [0, 1, 63, 64, 300]), (64, 16, 3, [1, 0, 17, 200, 15], [5, 9, 0, 31, 16]), (128, 256, 2, [513], [255]),
    (64, 32, 1, [64, 1, 127, 2], [0, 31, 1, 62]), (128, 128, 4, [33, 1, 90], [100, 0, 127])])
def test_append_writes_what_the_definition_says_and_nothing_else(A, bits, width, page, heads, counts, prefix):
    import torch
    lengths = [p + n for p, n in zip(prefix, counts)]
    table, pages = plan_pages(lengths, page, 3)
    cache = A.KVCache.empty(pages, heads, page, width, bits)
    for x in (cache.k, cache.v, cache.k_scale, cache.v_scale):
        if x is not None:
            x.view(torch.uint8).fill_(0x5A)
    T = sum(counts)
    fused = randn(T + width + bits, T, 2 * heads, width) * 3
    fused[0] = 1.25                                        # constant rows
    fused[T // 2, :, 5] = 80.0                             # an outlier
    fused[T - 1] = fused[T - 1].abs() + 40                 # zero outside the range
    k, v = fused[:, :heads], fused[:, heads:]
    start = np.concatenate([[0], np.cumsum(counts)])
    before = [None if x is None else x.cpu().clone() for x in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    held = A.append(cache, k, v, i32(start), i32(prefix), i32(table), values=bits != 16)
    kn, vn = k.float().cpu().numpy(), v.float().cpu().numpy()
    want = [None if x is None else x.float().numpy() if x.dtype == torch.bfloat16 else x.numpy() for x in before]
    for b, n in enumerate(counts):
        for i in range(n):
            pos, t = prefix[b] + i, start[b] + i
            p, s = table[b, pos // page], pos % page
            if bits == 16:
                want[0][p, :, s], want[1][p, :, :, s] = kn[t], vn[t]
                continue
            for j, rows in enumerate((kn[t], vn[t])):
                code, step, offset = quantise32(rows, bits)
                if j == 0:
                    want[0][p, :, s] = pack(code, bits)
                else:
                    want[1][p, :, :, s] = pack(code, bits)
                want[2 + j][p, :, s, 0], want[2 + j][p, :, s, 1] = step[:, 0], offset[:, 0]
    got = [cache.k, cache.v, cache.k_scale, cache.v_scale]
    for x, w in zip(got, want):
        if x is not None:
            x = x.float().cpu().numpy() if x.dtype == torch.bfloat16 else x.cpu().numpy()
            assert np.array_equal(x, w, equal_nan=True)
    if bits != 16:
        for rows, value in ((kn, held[0]), (vn, held[1])):
            code, step, offset = quantise32(rows, bits)
            exact = step.astype(np.float64) * code + offset
            # the product and the sum in 32 bits, then one rounding to bf16
            assert np.all(np.abs(value.double().cpu().numpy() - exact) <= V * np.abs(exact) + 2.0 ** -23 * (np.abs(step * code) + np.abs(offset)))


def test_append_drops_tokens_without_a_place(A):
    """Beyond the table's row, on pages that do not exist, rows of no sequence, counts below zero: nothing is written for them."""
    import torch
    cache = A.KVCache.empty(3, 1, 16, 64, 16)
    cache.k.zero_(), cache.v.zero_()
    k, v = randn(1, 40, 1, 64), randn(2, 40, 1, 64)
    table = i32([[0, 7], [-3, 1]])
    A.append(cache, k, v, i32([0, 20, 35]), i32([20, 10]), table)       # b0: 16 beyond the row and 12 on page 7; b1: 6 on page -3, 9 on page 1
    want = torch.zeros_like(cache.k)
    want[1, 0, :9] = k[26:35, 0]
    assert torch.equal(cache.k, want)
    assert torch.equal(cache.v[1, 0, :, :9], v[26:35, 0].t()) and torch.all(cache.v[0] == 0) and torch.all(cache.v[1, 0, :, 9:] == 0)
    cache.k.zero_()
    A.append(cache, k, v, i32([30, 20, 1000]), i32([0, -5]), i32([[0, 1], [2, 2]]))   # a falling start; a start and a prefix out of range
    assert torch.all(cache.k[:2] == 0)
    A.append(cache, k[:0], v[:0], i32([0, 0]), i32([0]), i32([[0]]))


def test_append_of_unaligned_rows(A):
    import torch
    for bits in (16, 8, 4):
        cache, other = A.KVCache.empty(4, 2, 32, 64, bits), A.KVCache.empty(4, 2, 32, 64, bits)
        for c in (cache, other):
            for x in (c.k, c.v, c.k_scale, c.v_scale):
                if x is not None:
                    x.view(torch.uint8).fill_(0)
        x = randn(5, 50 * 300)[1:].as_strided((50, 4, 64), (297, 67, 1))
        start, prefix, table = i32([0, 50]), i32([9]), i32([[3, 1]])
        room = torch.zeros(50 * 300, dtype=torch.bfloat16, device="cuda:0")
        out = room[3:].as_strided((50, 4, 64), (297, 67, 1))
        more = {} if bits == 16 else dict(values=True, k_values=out[:, :2], v_values=out[:, 2:])
        A.append(cache, x[:, :2], x[:, 2:], start, prefix, table, **more)
        held = A.append(other, x[:, :2].contiguous(), x[:, 2:].contiguous(), start, prefix, table, values=bits != 16)
        for a, b in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), (other.k, other.v, other.k_scale, other.v_scale)):
            assert a is None or torch.equal(a, b)
        if bits != 16:
            assert torch.equal(out[:, :2], held[0]) and torch.equal(out[:, 2:], held[1])


# ------------------------------------------------------------------------------------------------ attention

def values_of(cache, which, table, length):
    """Keys or values of one sequence in 64 bits, [heads, length, width], and the magnitude of their terms."""
    import torch
    pool, scale = (cache.k, cache.k_scale) if which == "k" else (cache.v.transpose(2, 3), cache.v_scale)
    pages = torch.from_numpy(np.where((table >= 0) & (table < cache.pages), table, 0).astype(np.int64)).to(pool.device)[:(length + cache.page_tokens - 1) // cache.page_tokens]
    x = pool[pages]
    if cache.bits == 4:
        x = torch.cat([x & 15, x >> 4], -1)
    x = x.double()
    terms = torch.zeros_like(x[..., 0])
    if cache.bits != 16:
        step, offset = scale[pages][..., :1].double(), scale[pages][..., 1:].double()
        x = x * step + offset
        terms = (256 * step.abs() + offset.abs())[..., 0]
    return x.transpose(0, 1).flatten(1, 2)[:, :length], terms.transpose(0, 1).flatten(1, 2)[:, :length]


def attend64(q, cache, start, prefix, table, masks, scale, context=None):
    """(result, its bound without the result's own rounding), rows of no sequence zero."""
    import torch
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    size = torch.zeros_like(out)
    group = q.shape[1] // cache.heads
    for b in range(len(prefix)):
        n = start[b + 1] - start[b]
        length = prefix[b] + n
        length = min(length, table.shape[1] * cache.page_tokens, context if context is not None else length)
        (k, _), (v, terms) = values_of(cache, "k", table[b], length), values_of(cache, "v", table[b], length)
        seen = torch.zeros(n, length, dtype=torch.bool)
        for i in range(n):
            seen[i, :min(prefix[b], length)] = True
            for j in range(n):
                if prefix[b] + j < length and (masks[start[b] + i] >> j & 1 if masks is not None else j <= i):
                    seen[i, prefix[b] + j] = True
        for t in range(length):
            p = table[b, t // cache.page_tokens]
            if p < 0 or p >= cache.pages:
                seen[:, t] = False
        seen = seen.to(q.device)
        for h in range(q.shape[1]):
            rows = q[start[b]:start[b + 1], h].double()
            s = (rows @ k[h // group].t().contiguous() * scale).masked_fill(~seen, -math.inf)
            for i in range(n):
                pick = seen[i]
                if not pick.any():
                    continue
                w = torch.softmax(s[i, pick], 0)
                out[start[b] + i, h] = w @ v[h // group][pick]
                size[start[b] + i, h] = 1.25 * V * (w @ v[h // group][pick].abs()) + 2.0 ** -22 * (w @ terms[h // group][pick])
    return out, size


def tree_masks(n, seed):
    rng = np.random.default_rng(seed)
    masks = []
    for i in range(n):
        masks.append((masks[rng.integers(0, i)] if i else 0) | 1 << i)
    return masks


def signed(masks):
    import torch
    return torch.tensor([m - (1 << 64) if m >> 63 else m for m in masks], dtype=torch.int64, device="cuda:0")


def filled_cache(A, lengths, page, heads, width, bits, seed, garbage=True):
    """A cache holding random tokens, put there by `append`; what no token lies in is NaN (16 bits) or has NaN for its pair."""
    import torch
    table, pages = plan_pages(lengths, page, seed)
    cache = A.KVCache.empty(pages, heads, page, width, bits)
    for x in (cache.k, cache.v, cache.k_scale, cache.v_scale):
        if x is not None:
            x.view(torch.uint8).fill_(0xFF if garbage else 0)
    T = sum(lengths)
    k, v = randn(seed + 1, T, heads, width), randn(seed + 2, T, heads, width)
    k[..., 1] *= 6
    v[..., 7] *= 5
    A.append(cache, k, v, i32(np.concatenate([[0], np.cumsum(lengths)])), i32([0] * len(lengths)), i32(table))
    return cache, table


TREES = [  # width, page, cache heads, group, counts, prefix
    (128, 64, 2, 4, [1, 1, 1], [0, 1, 777]),
    (64, 16, 1, 1, [1, 2, 3], [15, 16, 0]),
    (128, 32, 3, 7, [5, 1, 64], [100, 2000, 31]),
    (128, 128, 1, 8, [48, 48], [1000, 4097]),
    (64, 256, 2, 64, [1, 2], [300, 255]),
    (64, 64, 4, 2, [17, 33, 9], [63, 64, 65]),
    (128, 16, 1, 3, [64], [9000]),
    (64, 32, 8, 4, [1] * 9, [0, 5, 17, 64, 128, 255, 256, 257, 3000]),
]


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("case", TREES, ids=str)
def test_tree_attention(A, case, bits):
    import torch
    width, page, heads, group, counts, prefix = case
    lengths = [p + n for p, n in zip(prefix, counts)]
    cache, table = filled_cache(A, lengths, page, heads, width, bits, 11)
    start = [0] + list(np.cumsum(counts))
    T = start[-1]
    q = randn(21, T, heads * group, width)
    masks = [m for b, n in enumerate(counts) for m in tree_masks(n, b)]
    scale = width ** -0.5
    for mask, ref in ((signed(masks), masks), (None, None)):
        want, size = attend64(q, cache, start, prefix, table, ref, scale)
        for context in (max(lengths), None):
            got = A.tree_attention(q, cache, i32(start), i32(prefix), i32(table), mask=mask, max_query=max(counts), max_context=context)
            within(got, want, size)
            assert torch.equal(got, A.tree_attention(q, cache, i32(start), i32(prefix), i32(table), mask=mask, max_query=max(counts), max_context=context))


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_rows_that_see_nothing_and_what_is_hidden(A, bits):
    """Empty masks, empty sequences, and infinities and NaNs in places that a row does not see."""
    import torch
    width, page, heads, group = 128, 32, 2, 4
    counts, prefix = [4, 0, 6, 1], [0, 50, 70, 0]
    lengths = [p + n for p, n in zip(prefix, counts)]
    start = [0, 4, 4, 10, 11]
    masks = [0, 1, 0b0110, 0b1001] + [0b111111, 0b000001, 0b000100, 0b001000, 0, 0b100001] + [0]
    q = randn(5, 11, heads * group, width)
    cache, table = filled_cache(A, lengths, page, heads, width, bits, 4)
    call = dict(mask=signed(masks), max_query=6)
    want, size = attend64(q, cache, start, prefix, table, masks, width ** -0.5)
    got = A.tree_attention(q, cache, i32(start), i32(prefix), i32(table), **call)
    within(got, want, size)
    assert torch.all(got[0] == 0) and torch.all(got[10] == 0)                    # nothing seen
    # new token 3 of sequence 2 (seen by its tokens 0 and 3) holds what must not reach the others
    p, s = int(table[2, 73 // page]), 73 % page
    for bad in (math.nan, math.inf):
        if bits == 16:
            cache.k[p, :, s], cache.v[p, :, 5:9, s] = bad, bad
        else:
            cache.k_scale[p, :, s], cache.v_scale[p, :, s] = bad, bad
        other = A.tree_attention(q, cache, i32(start), i32(prefix), i32(table), **call)
        hidden = [i for i in range(11) if i not in (4, 7)]
        assert torch.equal(other[hidden], got[hidden])
        assert not torch.isfinite(other[[4, 7]][..., 5:9]).any()
    if bits == 16:      # values alone: the entries that hold them, in the rows that see them
        cache, table = filled_cache(A, lengths, page, heads, width, bits, 4)
        p, s = int(table[2, 73 // page]), 73 % page
        cache.v[p, 1, 5, s], cache.v[p, 0, 100, s] = -math.inf, math.nan
        other = A.tree_attention(q, cache, i32(start), i32(prefix), i32(table), **call)
        wrong = torch.zeros_like(other, dtype=torch.bool)
        wrong[[4, 7], group:, 5] = True
        assert torch.all(other[wrong] == -math.inf)
        nans = torch.zeros_like(wrong)
        nans[[4, 7], :group, 100] = True
        assert torch.all(torch.isnan(other[nans]))
        assert torch.equal(other[~(wrong | nans)], got[~(wrong | nans)])


def test_infinities_that_are_seen(A):
    """A visible score of +inf or NaN makes its row NaN, one of -inf weighs nothing; other rows keep their results."""
    import torch
    heads, width, page = 1, 64, 32
    cache, table = filled_cache(A, [200], page, heads, width, 16, 8)
    q = randn(3, 2, 1, width).abs()
    start, prefix = i32([0, 2]), i32([198])
    base = A.tree_attention(q, cache, start, prefix, i32(table), max_query=2)
    at = (int(table[0, 70 // page]), 0, 70 % page)
    row = cache.k[at].clone()
    cache.k[at] = math.inf
    assert torch.isnan(A.tree_attention(q, cache, start, prefix, i32(table), max_query=2)).all()
    cache.k[at] = -math.inf
    got = A.tree_attention(q, cache, start, prefix, i32(table), max_query=2)
    cache.k[at] = row
    table2 = table.copy()
    seen = torch.ones(200, dtype=torch.bool, device="cuda:0")
    seen[70] = False
    k, v = values_of(cache, "k", table2[0], 200)[0][0], values_of(cache, "v", table2[0], 200)[0][0]
    for i in range(2):
        pick = seen.clone()
        pick[199 if i == 0 else 200:] = False
        w = torch.softmax(k[pick] @ q[i, 0].double() * width ** -0.5, 0)
        within(got[i, 0], w @ v[pick], 1.25 * V * (w @ v[pick].abs()))
    assert torch.equal(A.tree_attention(q, cache, start, prefix, i32(table), max_query=2), base)


@pytest.mark.parametrize("bits", [16, 4])
def test_scales_large_scores_and_strides(A, bits):
    """Peaked and negative scales, scores far beyond what an exponential holds, rows in slices of a fused tensor, results in place."""
    import torch
    counts, prefix = [3, 40], [600, 77]
    cache, table = filled_cache(A, [603, 117], 64, 2, 128, bits, 2)
    start = [0, 3, 43]
    masks = tree_masks(3, 0) + tree_masks(40, 1)
    fused = randn(6, 43, 20, 128)
    q = fused[:, 3:11]
    args = (cache, i32(start), i32(prefix), i32(table))
    for scale, by in ((None, 1.0), (-0.3, 1.0), (2.0, 1.0), (0.0, 1.0)):
        want, size = attend64(q, cache, start, prefix, table, masks, 128 ** -0.5 if scale is None else scale)
        got = A.tree_attention(q, *args, mask=signed(masks), max_query=40, scale=scale)
        # scores of up to some 100 are rounded to 32 bits: 2^-17 in the weights, within the quarter; at 2.0 they reach 300
        within(got, want, size)
    odd = torch.empty(43 * 1300 + 9, dtype=torch.bfloat16, device="cuda:0")[1:].as_strided((43, 8, 128), (1291, 131, 1))
    odd.copy_(q)
    base = A.tree_attention(q, *args, mask=signed(masks), max_query=40)
    assert torch.equal(A.tree_attention(odd, *args, mask=signed(masks), max_query=40), base)
    out = A.tree_attention(odd, *args, mask=signed(masks), max_query=40, out=odd)
    assert out is odd and torch.equal(odd, base)


def test_bounds_of_the_arguments_on_the_device(A):
    """Pages that do not exist are not seen, a context beyond max_context neither, rows beyond max_query get no result."""
    import torch
    cache, table = filled_cache(A, [500], 32, 1, 64, 16, 9)
    q = randn(3, 6, 2, 64)
    start, prefix = [0, 4], [496]
    holes = table.copy()
    holes[0, 2], holes[0, 9] = -1, 1 << 30
    want, size = attend64(q[:4], cache, start, prefix, holes, None, 0.125)
    got = torch.full_like(q, 9.0)
    A.tree_attention(q, cache, i32(start), i32(prefix), i32(holes), max_query=4, out=got)
    within(got[:4], want, size)
    assert torch.all(got[4:] == 9.0)                                              # rows of no sequence
    want, size = attend64(q[:4], cache, start, prefix, table, None, 0.125, context=300)
    within(A.tree_attention(q, cache, i32(start), i32(prefix), i32(table), max_query=4, max_context=300)[:4], want, size)
    got.fill_(9.0)
    A.tree_attention(q, cache, i32(start), i32(prefix), i32(table), max_query=2, out=got)
    want, size = attend64(q[:4], cache, start, prefix, table, None, 0.125)
    within(got[:2], want[:2], size[:2])
    assert torch.all(got[2:] == 9.0)
    A.tree_attention(q, cache, i32([3, 1]), i32([-9]), i32(table), max_query=2, out=got)   # a count below zero: no row
    assert A.tree_attention(q[:0], cache, i32([0, 0]), i32([5]), i32(table)).shape == (0, 2, 64)


@pytest.mark.parametrize("bits", [16, 4])
def test_caches_beyond_32_bit_offsets(A, bits):
    """Pages whose entries lie past 2^32 bytes of the pool."""
    import torch
    heads, page, width = 8, 256, 128
    per_page = heads * page * width * 2 if bits == 16 else heads * page * width // 2
    pages = (1 << 32) // per_page + 40
    cache = A.KVCache.empty(pages, heads, page, width, bits)
    lengths, counts = [700, 1300], [3, 1]
    table = np.array([[pages - 1, pages - 9, 5, 0, 0, 0], [pages - 20, 1, pages - 3, pages - 2, pages - 30, pages - 31]], np.int32)
    k, v = randn(1, 2000, heads, width), randn(2, 2000, heads, width)
    A.append(cache, k, v, i32([0, 700, 2000]), i32([0, 0]), i32(table))
    q = randn(3, 4, 16, width)
    start, prefix = [0, 3, 4], [697, 1299]
    want, size = attend64(q, cache, start, prefix, table, None, width ** -0.5)
    got = A.tree_attention(q, cache, i32(start), i32(prefix), i32(table), max_query=3, max_context=1300)
    within(got, want, size)
    if bits == 16:
        assert torch.equal(cache.k[pages - 1, :, 17], k[17]) and torch.equal(cache.v[pages - 2, :, :, 0], v[700 + 768])


def test_on_another_stream_and_in_a_graph(A):
    """The calls follow the current stream, and a captured decode step gives the eager result on every replay."""
    import torch
    T, heads, group, width = 3, 2, 4, 128
    plan = A.Rotary(width)
    wq, wk = 1 + randn(1, width) / 4, 1 + randn(2, width) / 4

    def step(cache, fused, pos, start, prefix, table, mask):
        q, k, v = fused[:, :heads * group], fused[:, heads * group:heads * (group + 1)], fused[:, heads * (group + 1):]
        q, k = A.qk_norm_rotary(plan, q, k, wq, wk, pos)
        A.append(cache, k, v, start, prefix, table)
        return A.tree_attention(q, cache, start, prefix, table, mask=mask, max_query=1, max_context=2000)

    lengths = [1500, 1, 700]
    fused = randn(5, T, heads * (group + 2), width)
    pos, start, prefix = torch.tensor([n - 1 for n in lengths], device="cuda:0"), i32([0, 1, 2, 3]), i32([n - 1 for n in lengths])
    mask = signed([1, 1, 1])
    cache, table = filled_cache(A, lengths, 64, heads, width, 4, 3)
    table = i32(table)
    base = step(cache, fused, pos, start, prefix, table, mask)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device="cuda:0")
    with torch.cuda.stream(side):
        for _ in range(4):
            big = big @ big / 4096                          # keeps the side stream busy before the inputs are there
        late = fused * 0
        late += fused
        other = step(cache, late, pos, start, prefix, table, mask)
    side.synchronize()
    assert torch.equal(other, base)
    graph = torch.cuda.CUDAGraph()
    held = fused.clone()
    with torch.cuda.graph(graph):
        out = step(cache, held, pos, start, prefix, table, mask)
    for seed in range(4):
        held.copy_(randn(30 + seed, T, heads * (group + 2), width))
        graph.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        assert torch.equal(replayed, step(cache, held, pos, start, prefix, table, mask))


def test_a_graph_keeps_its_workspace(A):
    """A larger call on the capturing stream, which takes a larger workspace, leaves a captured call's results alone."""
    import torch
    heads, width = 2, 128
    cache, table = filled_cache(A, [3000, 3000], 64, heads, width, 16, 3)
    start, prefix, table = i32([0, 1, 2]), i32([2999, 2999]), i32(table)
    q = randn(4, 2, 8, width)
    base = A.tree_attention(q, cache, start, prefix, table)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        out = A.tree_attention(q, cache, start, prefix, table)
    more = randn(5, 128, 64, width)
    for _ in range(3):
        with torch.cuda.stream(side):
            A.tree_attention(more, cache, i32([0, 64, 128]), i32([2936, 2936]), table)
            out.zero_()
            graph.replay()
        torch.cuda.synchronize()
        held = [torch.full((1 << 22,), 3.0, device="cuda:0") for _ in range(8)]       # takes whatever was given back
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, base) and all(torch.all(x == 3.0) for x in held)


# ------------------------------------------------------------------------------------------------ refusals

def test_refusals(A):
    import torch
    from paper_2605_10793_amd import binding
    plan = A.Rotary(128)
    q, k = randn(1, 4, 2, 128), randn(2, 4, 1, 128)
    pos = torch.arange(4, device="cuda:0")
    w = randn(3, 128)
    with pytest.raises(ValueError):
        A.Rotary(128, scaling="other")
    for bad in (dict(part=7), dict(part=0), dict(part=514), dict(part=64, theta=1.0), dict(part=64, scaling="linear", factor=0.5),
                dict(part=64, scaling="bands", factor=2.0, low=4.0, high=4.0), dict(part=2, scaling="base", factor=2.0)):
        with pytest.raises(binding.ConqurError):
            A.Rotary(**bad)
    for call in (lambda: A.rotary(plan, q.half(), pos), lambda: A.rotary(plan, q.cpu(), pos), lambda: A.rotary(plan, q, pos.int()),
                 lambda: A.rotary(plan, q, pos[:3]), lambda: A.rotary(plan, q, pos, k=k.float()), lambda: A.rotary(plan, q.transpose(1, 2), pos),
                 lambda: A.rotary(plan, q, pos, out=k), lambda: A.qk_norm_rotary(plan, q, k, w[:64], w, pos),
                 lambda: A.qk_norm_rotary(plan, q, k, w.float(), w, pos)):
        with pytest.raises(ValueError):
            call()
    same = torch.empty(128, device="cuda:0", dtype=torch.bfloat16)
    for call in (lambda: A.rotary(plan, q[..., :64].contiguous(), pos), lambda: A.rotary(plan, q, pos, out=same.as_strided((4, 2, 128), (0, 0, 1))),
                 lambda: A.qk_norm_rotary(plan, q, k, w, w, pos, eps=-1.0), lambda: A.qk_norm_rotary(plan, q, k, w, w, pos, eps=math.nan)):
        with pytest.raises(binding.ConqurError) as e:
            call()
        assert e.value.status == binding.EINVAL
    cache = A.KVCache.empty(2, 1, 64, 128)
    start, prefix, table = i32([0, 4]), i32([0]), i32([[0]])
    for call in (lambda: A.KVCache(cache.k, cache.k), lambda: A.KVCache(cache.k, cache.v, bits=8), lambda: A.KVCache(cache.k, cache.v, bits=5),
                 lambda: A.KVCache(cache.k.to(torch.uint8), cache.v.to(torch.uint8), bits=8),
                 lambda: A.append(cache, q, k, start, prefix, table), lambda: A.append(cache, k, k.float(), start, prefix, table),
                 lambda: A.append(cache, k, k, start[:1], prefix, table), lambda: A.append(cache, k, k, start.long(), prefix, table),
                 lambda: A.append(cache, k, k, start, prefix, table.long()), lambda: A.tree_attention(q.float(), cache, start, prefix, table),
                 lambda: A.tree_attention(q[..., :64], cache, start, prefix, table), lambda: A.tree_attention(q, cache, start, prefix, table, mask=start),
                 lambda: A.tree_attention(q, cache, start, prefix, table, out=k)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: A.append(cache, k, k, start, prefix, table, values=True),            # 16 bits hold the values themselves
                 lambda: A.append(A.KVCache.empty(2, 1, 48, 128), k, k, start, prefix, table),
                 lambda: A.append(A.KVCache.empty(2, 1, 8, 128), k, k, start, prefix, table),
                 lambda: A.append(A.KVCache.empty(2, 1, 64, 96), k[..., :96], k[..., :96], start, prefix, table),
                 lambda: A.tree_attention(q, cache, start, prefix, table, max_query=0), lambda: A.tree_attention(q, cache, start, prefix, table, max_query=65),
                 lambda: A.tree_attention(q, cache, start, prefix, table, scale=math.inf),
                 lambda: A.tree_attention(randn(1, 4, 3, 128), A.KVCache.empty(2, 2, 64, 128), start, prefix, table),
                 lambda: A.tree_attention(randn(1, 4, 65, 128), cache, start, prefix, table)):
        with pytest.raises(binding.ConqurError) as e:
            call()
        assert e.value.status == binding.EINVAL
