"""Attention of packed sequences where values are not finite, rows lie anywhere, streams and graphs differ."""
import math

import pytest
import torch

from attention_reference import attend, close, seen_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def case(counts, heads=4, kv=2, width=64, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    tokens = sum(counts)
    q = torch.randn(tokens, heads, width, device=DEV, generator=g).to(torch.bfloat16)
    k, v = (torch.randn(tokens, kv, width, device=DEV, generator=g).to(torch.bfloat16) for _ in range(2))
    grad = torch.randn(tokens, heads, width, device=DEV, generator=g).to(torch.bfloat16)
    start = torch.tensor([sum(counts[:b]) for b in range(len(counts) + 1)], dtype=torch.int32, device=DEV)
    return q, k, v, grad, start


def both(q, k, v, grad, start, **options):
    from paper_2605_10793_amd import attention as A
    out, lse = A.attention(q, k, v, start, lse=True, **options)
    return (out, *A.attention_backward(q, k, v, out, lse, grad, start, **options))


@pytest.mark.parametrize("width", [64, 80, 128])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("biased", [False, True])
def test_documents_and_padding_do_not_meet(width, value, biased):
    """A document among others, and padding, hold what is not finite; the others' results are as without it, padding's are zeros."""
    n, edges = 230, [0, 50, 130, 205]
    q, k, v, grad, start = case([n], width=width)
    first = torch.zeros(n, dtype=torch.int32)
    last = torch.zeros(n, dtype=torch.int32)
    for a, b in zip(edges, edges[1:]):
        first[a:b], last[a:b] = a, torch.arange(a + 1, b + 1, dtype=torch.int32)
    options = dict(first=first.to(DEV), last=last.to(DEV), cap=20.0 if biased else 0.0, slopes=torch.full((4,), 0.1, device=DEV) if biased else None)
    clean = both(q, k, v, grad, start, **options)
    for which in range(4):
        bad = [x.clone() for x in (q, k, v, grad)]
        bad[which][50:130:7] = value
        bad[which][205:] = value
        got = both(*bad, start, **options)
        for x, y in zip(got, clean):
            assert torch.equal(x[:50], y[:50]) and torch.equal(x[130:205], y[130:205])
            assert not x[205:].any()
    bad = [x.clone() for x in (q, k, v, grad)]
    for x in bad:
        x[205:] = value
    got = both(*bad, start, **options)
    for x, y in zip(got, clean):
        assert torch.equal(x, y)


@pytest.mark.parametrize("width", [64, 128])
def test_later_tokens_do_not_reach_earlier_ones(width):
    n, t = 200, 77
    q, k, v, grad, start = case([n], width=width)
    clean = both(q, k, v, grad, start)
    for which in (1, 2):
        bad = [x.clone() for x in (q, k, v, grad)]
        bad[which][t, 0, 3] = math.nan
        got = both(*bad, start)
        for i in (0, 1):          # the result and the queries' gradients: of the rows that see the key, all of two heads
            assert torch.equal(got[i][:t], clean[i][:t])
            assert torch.equal(got[i][:, 2:], clean[i][:, 2:])
        assert bool(torch.isnan(got[0][t:, :2, 3]).all()) and bool(torch.isnan(got[1][t:, :2]).all())
    # queries and gradients: rows that do not see a key leave its gradients alone
    for which in (0, 3):
        bad = [x.clone() for x in (q, k, v, grad)]
        bad[which][t, 0] = math.nan
        got = both(*bad, start)
        for i in (2, 3):
            assert torch.equal(got[i][t + 1:], clean[i][t + 1:])
            assert torch.equal(got[i][:, 1], clean[i][:, 1])
            assert bool(torch.isnan(got[i][:t + 1, 0]).all())


def test_infinite_values():
    """An infinity among the values reaches the entry it stands in, of the rows that see it."""
    from paper_2605_10793_amd import attention as A
    n, t = 150, 40
    q, k, v, _, start = case([n], heads=2, kv=1)
    clean = A.attention(q, k, v, start)
    v = v.clone()
    v[t, 0, 5], v[t, 0, 6], v[t + 1, 0, 6], v[t, 0, 7] = math.inf, math.inf, -math.inf, math.nan
    got = A.attention(q, k, v, start)
    assert torch.equal(got[:t], clean[:t])
    assert bool((got[t:, :, 5] == math.inf).all()) and bool(torch.isnan(got[t + 1:, :, 6]).all()) and bool(torch.isnan(got[t:, :, 7]).all())
    assert bool(torch.isfinite(got[:, :, [0, 4, 8, 40]]).all())


def test_scores_of_minus_infinity():
    """A row whose every score is -inf gets zeros; a single such score has no weight."""
    q, k, v, grad, start = case([70], heads=1, kv=1)
    q.abs_()
    k[0] = -math.inf
    k[1] = 1.0
    out, dq, dk, dv = both(q, k, v, grad, start)
    assert not out[0].any() and torch.equal(out[1, 0], v[1, 0])
    assert bool(torch.isfinite(out).all())


@pytest.mark.parametrize("width", [64, 80, 128])
@pytest.mark.parametrize("t", [0, 40, 99])
def test_gradients_of_scores_of_minus_infinity(width, t):
    """A key whose scores are all -inf, in the first of two documents: its rows and what they see have the gradients that they would have without it, or NaN (0 times
    an infinity); rows before it, and the other document and sequence, have those of a call without it, bit by bit."""
    n, edge, scale = 170, 100, width ** -0.5
    q, k, v, grad, start = case([n, 30], heads=2, kv=1, width=width, seed=t)
    q.abs_()
    place = torch.arange(n + 30)
    first = torch.where(place < edge, 0, torch.where(place < n, edge, 0)).to(torch.int32)
    last = (torch.where(place < n, place, place - n) + 1).to(torch.int32)
    options = dict(first=first.to(DEV), last=last.to(DEV))
    clean = both(q, k, v, grad, start, **options)
    k[t] = -math.inf
    out, dq, dk, dv = both(q, k, v, grad, start, **options)
    assert bool(torch.isfinite(out).all()) and (t or not out[0].any())
    for x, y in zip((out, dq), clean):
        assert torch.equal(x[:t], y[:t])
    for x, y in zip((out, dq, dk, dv), clean):
        assert torch.equal(x[edge:], y[edge:])
    seen = seen_of(edge, None, None, 0)
    seen[:, t] = False
    finite = k[:edge].clone()
    finite[t] = 0
    want = attend(q[:edge].cpu(), finite.cpu(), v[:edge].cpu(), seen, place[:edge], scale, grad=grad[:edge].cpu())
    close(out[:edge], want["out"], want["out_tol"], "out")
    for name, x in (("dq", dq), ("dk", dk), ("dv", dv)):
        nan = torch.isnan(x[:edge]).cpu()
        close(torch.where(nan, want[name], x[:edge].cpu().double()), want[name], want[name + "_tol"], name)


@pytest.mark.parametrize("how", ["odd strides", "unaligned", "heads first", "one row for all"])
def test_rows_anywhere(how):
    """Rows that do not start at multiples of 16 bytes, heads that lie further apart than tokens, broadcast rows."""
    from paper_2605_10793_amd import attention as A
    n, heads, kv, width = 90, 4, 2, 80
    q, k, v, grad, start = case([50, 40], heads, kv, width)
    plain = both(q, k, v, grad, start)

    def moved(x):
        t, h, w = x.shape
        if how == "odd strides":
            y = torch.empty(t, h, w + 5, dtype=x.dtype, device=DEV)[..., :w]
        elif how == "unaligned":
            y = torch.empty(t * h * w + 1, dtype=x.dtype, device=DEV)[1:].view(t, h, w)
        elif how == "heads first":
            y = torch.empty(h, t, w, dtype=x.dtype, device=DEV).transpose(0, 1)
        else:
            return x
        return y.copy_(x)
    if how == "one row for all":
        k, v = k[:1].expand(n, kv, width), v[:, :1].expand(n, kv, width)
        q, grad = q[:, :1].expand(n, heads, width), grad[:1, :1].expand(n, heads, width)
        plain = both(q.contiguous(), k.contiguous(), v.contiguous(), grad.contiguous(), start)
    got = both(*(moved(x) for x in (q, k, v, grad)), start)
    for x, y in zip(got, plain):
        assert torch.equal(x, y)
    out = moved(torch.zeros_like(plain[0])) if how != "one row for all" else torch.zeros_like(plain[0])
    A.attention(q, k, v, start, out=out)
    assert torch.equal(out, plain[0])


def test_out_over_q_and_rows_of_no_sequence():
    from paper_2605_10793_amd import attention as A
    q, k, v, _, start = case([60])
    start = torch.tensor([7, 40, 52], dtype=torch.int32, device=DEV)
    want = A.attention(q, k, v, start)
    mine = q.clone()
    A.attention(mine, k, v, start, out=mine)
    assert torch.equal(mine[7:52], want[7:52]) and torch.equal(mine[:7], q[:7]) and torch.equal(mine[52:], q[52:])


def test_starts_out_of_range():
    """Starts beyond the rows, and such as fall, touch nothing that is not there."""
    from paper_2605_10793_amd import attention as A
    q, k, v, grad, _ = case([64])
    for start in ([-5, 30, 1000], [0, 0, 0], [64, 64], [100, 200], [0, 64, 64, 64]):
        start = torch.tensor(start, dtype=torch.int32, device=DEV)
        out, dq, dk, dv = both(q, k, v, grad, start)
        clamped = start.clamp(0, 64)
        want, *grads = both(q, k, v, grad, clamped)
        assert torch.equal(out, want) and all(torch.equal(x, y) for x, y in zip((dq, dk, dv), grads))
    A.attention(q, k, v, torch.tensor([0, 50, 20, 64], dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()


def test_gradients_against_differences():
    """sum(out * grad) moves with each input as its gradient says.  Central differences of the 64-bit formula around bf16 inputs, along random directions: the
    directional derivative is off by no more than the gradients' own tolerances, added up with the direction."""
    counts, heads, kv, width = [40], 2, 1, 64
    q, k, v, grad, start = case(counts, heads, kv, width, seed=5)
    _, dq, dk, dv = both(q, k, v, grad, start, cap=5.0)
    seen = seen_of(40, None, None, 0)
    host = [x.double().cpu() for x in (q, k, v, grad)]
    want = attend(*host[:3], seen, torch.arange(40), width ** -0.5, 5.0, None, host[3])
    f = lambda x: float((attend(*x, seen, torch.arange(40), width ** -0.5, 5.0)["out"] * host[3]).sum())
    g = torch.Generator().manual_seed(1)
    for i, (got, name) in enumerate(((dq, "dq"), (dk, "dk"), (dv, "dv"))):
        way = torch.randn(host[i].shape, generator=g, dtype=torch.float64)
        step = 1e-4
        up, down = [list(host[:3]) for _ in range(2)]
        up[i], down[i] = host[i] + step * way, host[i] - step * way
        slope = (f(up) - f(down)) / (2 * step)
        size = float((want[name].abs() * way.abs()).sum())
        # (third derivatives: step^2 of the size of things; 64-bit sums over 2 step)
        assert abs(float((got.double().cpu() * way).sum()) - slope) <= float((want[name + "_tol"] * way.abs()).sum()) + 1e-5 * size


def test_streams_and_graphs():
    from paper_2605_10793_amd import attention as A
    q, k, v, grad, start = case([100, 333], heads=4, kv=4, width=128)
    want = both(q, k, v, grad, start)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = both(q, k, v, grad, start)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    sq, sk, sv, sg = (x.clone() for x in (q, k, v, grad))
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one = both(sq, sk, sv, sg, start)
    with torch.cuda.graph(other):
        two = both(sq, sk, sv, sg, start, window=30)
    for seed in range(3):
        fresh = case([100, 333], heads=4, kv=4, width=128, seed=seed + 10)
        for x, y in zip((sq, sk, sv, sg), fresh):
            x.copy_(y)
        graph.replay()
        other.replay()
        eager = both(*fresh[:4], start), both(*fresh[:4], start, window=30)
        torch.cuda.synchronize()
        for mine, theirs in zip((one, two), eager):
            assert all(torch.equal(x, y) for x, y in zip(mine, theirs))


def test_shared_keys_on_streams_in_graphs_and_in_place():
    """Calls whose keys several workgroups share: two under way at once, captured ones between eager ones, results over the queries, rows anywhere."""
    from paper_2605_10793_amd import attention as A
    counts = [1700]
    made = [case(counts, heads=2, kv=1, width=64, seed=s) for s in range(4)]
    want = [both(*x) for x in made]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in made]
    got = []
    for _ in range(3):
        for stream, x in zip(streams, made):
            with torch.cuda.stream(stream):
                got.append(both(*x))
    torch.cuda.synchronize()
    for i, x in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(x, want[i % len(made)]))
    sq, sk, sv, sg, start = (x.clone() for x in made[0])
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one = both(sq, sk, sv, sg, start)
    with torch.cuda.graph(other):
        two = both(sq, sk, sv, sg, start, cap=30.0)
    for i in (1, 2, 3):
        for x, y in zip((sq, sk, sv, sg), made[i]):
            x.copy_(y)
        graph.replay()
        other.replay()
        capped = both(*made[i], cap=30.0)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(one, want[i])) and all(torch.equal(x, y) for x, y in zip(two, capped))
    q, k, v, grad, start = made[0]
    over = q.clone()
    A.attention(over, k, v, start, out=over)
    odd = torch.zeros(q.numel() + 1, dtype=torch.bfloat16, device=DEV)[1:].view(q.shape).copy_(q)          # rows at multiples of 2 bytes
    into = torch.zeros(q.numel() + 3, dtype=torch.bfloat16, device=DEV)[3:].view(q.shape)
    A.attention(odd, k, v, start, out=into)
    assert torch.equal(over, want[0][0]) and torch.equal(into, want[0][0])
    assert all(torch.equal(x, y) for x, y in zip(both(odd, k, v, grad, start), want[0]))
