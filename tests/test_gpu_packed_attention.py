"""Attention of packed sequences and its gradients against 64 bits: lengths, masks, head layouts, strides, what is not finite."""
import math

import pytest
import torch

from attention_reference import attend, close, seen_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def lists(counts, kind):
    """first and last of every token, by a rule; None: causal."""
    if kind in ("causal", "window"):
        return None, None
    first, last = [], []
    for n in counts:
        for i in range(n):
            if kind == "documents":
                size, pad = max(1, n * 5 // 16), n // 9
                first.append(i // size * size if i < n - pad else 0)
                last.append(i + 1 if i < n - pad else 0)
            elif kind == "prefix":
                first.append(0)
                last.append(max(i + 1, n // 4))
            elif kind == "both":           # sees everything, also beyond the end
                first.append(-3)
                last.append(n + 7)
            elif kind == "holes":          # every third row sees nothing, others a stretch anywhere
                first.append(i * 7 % n)
                last.append(0 if i % 3 == 1 else i * 7 % n + 1 + i * 5 % n)
            elif kind == "far":            # tokens see what comes much later
                first.append(n - 1 - i)
                last.append(n)
    return first, last


def inputs(counts, heads, kv, width, seed, lead=0, behind=0, strided=True):
    """Rows cut from a fused projection's output (strided), with `lead` and `behind` rows of no sequence."""
    g = torch.Generator().manual_seed(seed)
    tokens = sum(counts) + lead + behind
    fused = torch.randn(tokens, heads + 2 * kv, width, generator=g) * torch.exp(0.5 * torch.randn(heads + 2 * kv, width, generator=g))
    fused = fused.to(torch.bfloat16)
    q, k, v = fused[:, :heads], fused[:, heads:heads + kv], fused[:, heads + kv:]
    grad = torch.randn(tokens, heads, width, generator=g).to(torch.bfloat16)
    at, start = lead, [lead]
    for n in counts:
        at += n
        start.append(at)
    dev = fused.to(DEV)
    on = [dev[:, :heads], dev[:, heads:heads + kv], dev[:, heads + kv:]] if strided else [x.contiguous().to(DEV) for x in (q, k, v)]
    return (q, k, v, grad), (*on, grad.to(DEV)), torch.tensor(start, dtype=torch.int32, device=DEV)


def check(counts, heads, kv, width, kind="causal", window=0, cap=0.0, biased=False, seed=0, lead=0, behind=0, scale=None, strided=True):
    from paper_2605_10793_amd import attention as A
    host, dev, start = inputs(counts, heads, kv, width, seed, lead, behind, strided)
    first, last = lists(counts, kind)
    slopes = torch.exp2(-8 * (1 + torch.arange(heads, dtype=torch.float32)) / heads) if biased else None
    pad = lambda x: None if x is None else torch.tensor([0] * lead + x + [0] * behind, dtype=torch.int32, device=DEV)
    options = dict(first=pad(first), last=pad(last), window=window, cap=cap, slopes=None if slopes is None else slopes.to(DEV), scale=scale)
    out, lse = A.attention(*dev[:3], start, lse=True, **options)
    dq, dk, dv = A.attention_backward(*dev[:3], out, lse, dev[3], start, **options)
    again = A.attention(*dev[:3], start, **options)
    assert torch.equal(again, out)
    at = lead
    for b, n in enumerate(counts):
        rows, mine = slice(at, at + n), slice(at - lead, at - lead + n)
        seen = seen_of(n, first and first[mine], last and last[mine], window)
        want = attend(*(x[rows] for x in host[:3]), seen, torch.arange(n), width ** -0.5 if scale is None else scale, cap, slopes, host[3][rows])
        for name, got in (("out", out), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
            close(got[rows], want[name], want[name + "_tol"], f"{name} of sequence {b}")
        at += n
    for x in (out, dq, dk, dv):
        assert not x[:lead].any() and not x[at:].any()
    assert bool((lse[:lead] == -math.inf).all()) and bool((lse[at:] == -math.inf).all())


@pytest.mark.parametrize("width", [32, 64, 80, 96, 128])
@pytest.mark.parametrize("counts", [[1], [33], [200], [1, 64, 0, 65, 3, 130]])
def test_causal(width, counts):
    check(counts, 4, 2, width, seed=width + len(counts))


@pytest.mark.parametrize("heads, kv", [(1, 1), (8, 8), (5, 1), (24, 4), (64, 1), (6, 2)])
def test_head_layouts(heads, kv):
    check([70, 41], heads, kv, 64, seed=heads)


@pytest.mark.parametrize("kind", ["documents", "prefix", "both", "holes", "far"])
@pytest.mark.parametrize("width", [64, 128])
def test_masks(kind, width):
    check([150, 1, 77, 260], 4, 2, width, kind=kind, seed=len(kind), lead=5, behind=9)


@pytest.mark.parametrize("window", [1, 2, 63, 64, 100, 1000])
def test_windows(window):
    check([300, 65], 4, 1, 64, window=window, seed=window)


@pytest.mark.parametrize("cap, biased, kind", [(20.0, False, "causal"), (0.0, True, "prefix"), (50.0, True, "documents"), (2.0, True, "far"), (0.5, False, "holes")])
@pytest.mark.parametrize("width", [80, 128])
def test_caps_and_slopes(cap, biased, kind, width):
    check([140, 97], 6, 2, width, kind=kind, cap=cap, biased=biased, seed=int(cap) + width, behind=3)


@pytest.mark.parametrize("scale", [-0.2, 0.0, 1.0])
def test_scales(scale):
    check([90], 2, 2, 64, scale=scale, cap=0.0, seed=3)
    check([90], 2, 2, 64, scale=scale, cap=30.0, seed=4)


def test_windows_with_bounds():
    check([280], 4, 2, 64, kind="prefix", window=50, seed=11)
    check([280], 4, 2, 64, kind="far", window=90, seed=12)


def test_long():
    check([1500], 2, 1, 128, seed=21)


def test_many_sequences():
    check([(i * 5) % 7 for i in range(300)], 2, 1, 64, seed=22)
    check([1] * 5000, 1, 1, 32, seed=23)


@pytest.mark.parametrize("n", [61, 62, 63, 64, 4030, 4094])
def test_counts_of_sequences(n):
    """Around those where a part's sequence is found in one read more: every sequence, the last one too, and the rows behind it."""
    check([1 + (i * 5) % 3 for i in range(n - 1)] + [70], 1, 1, 32, seed=n, lead=2, behind=70)


@pytest.mark.parametrize("counts, heads, kv, width, options", [
    ([1300, 0, 1100], 8, 1, 64, dict(kind="documents")), ([1200], 4, 2, 128, dict(kind="prefix", cap=20.0, lead=3, behind=200)),
    ([900, 5, 1500], 6, 1, 96, dict(kind="holes", biased=True)), ([1900], 3, 1, 32, dict(window=700)), ([2050], 2, 2, 80, dict(kind="far"))])
def test_rows_in_parts(counts, heads, kv, width, options):
    """Few keys and many rows: several workgroups share the rows of 64 keys."""
    check(counts, heads, kv, width, seed=sum(counts), **options)


def test_contiguous_rows():
    check([100, 30], 4, 4, 128, seed=24, strided=False)


@pytest.mark.parametrize("cap", [200.0, 4096.0])
def test_large_caps(cap):
    """Scores next to zero under a cap that is far from them: what is left of cap - 2 cap / (1 + e^(2 u / cap)) is off by cap 2^-23, twice that with the
    products before it, and the weights and their sum by so much of themselves."""
    from paper_2605_10793_amd import attention as A
    counts, heads, kv, width = [150, 70], 4, 2, 64
    host, dev, start = inputs(counts, heads, kv, width, 5)
    out, lse = A.attention(*dev[:3], start, cap=cap, lse=True)
    at = 0
    for n in counts:
        rows = slice(at, at + n)
        seen = seen_of(n, None, None, 0)
        want, free = (attend(*(x[rows] for x in host[:3]), seen, torch.arange(n), width ** -0.5, c) for c in (cap, 0.0))
        more = cap * 2.0 ** -22
        close(out[rows], want["out"], free["out_tol"] + 2 * more * host[2][rows].abs().max().double(), "out")
        close(lse[rows], want["lse"], free["lse_tol"] + more, "lse")
        at += n


@pytest.mark.parametrize("width", [32, 64, 80, 96, 128])
@pytest.mark.parametrize("counts, heads, kv", [([1300], 2, 1), ([1500, 1400], 2, 2)])
@pytest.mark.parametrize("kind, window, cap, biased", [("causal", 0, 0.0, False), ("both", 0, 0.0, True), ("holes", 0, 30.0, False), ("causal", 1290, 20.0, True)])
def test_few_rows_whose_keys_are_shared(width, counts, heads, kv, kind, window, cap, biased):
    """So few rows that several workgroups take parts of their keys, some of them none."""
    check(counts, heads, kv, width, kind=kind, window=window, cap=cap, biased=biased, seed=width, lead=5, behind=3, strided=width != 80)


def test_shared_keys_that_are_not_finite():
    """Reach the rows that see them and no others, in every part."""
    from paper_2605_10793_amd import attention as A
    n, heads, width = 2048, 2, 128
    (q, k, v, grad), _, start = inputs([n], heads, 1, width, 11)
    first = (torch.arange(n) // 1024 * 1024).to(torch.int32).to(DEV)

    def run(k, v, grad):
        k, v, grad = (x.to(DEV) for x in (k, v, grad))
        out, lse = A.attention(q.to(DEV), k, v, start, first=first, lse=True)
        return (out, *A.attention_backward(q.to(DEV), k, v, out, lse, grad, start, first=first))
    clean = run(k, v, grad)
    bad_k, bad_v, bad_grad = k.clone(), v.clone(), grad.clone()
    bad_v[1400, 0, 3] = math.nan
    out, *_ = run(k, bad_v, grad)
    assert torch.equal(out[:1400], clean[0][:1400]) and bool(out[1400:, :, 3].isnan().all()) and not bool(out[1400:, :, 4].isnan().any())
    bad_k[1200] = math.inf
    out, dq, _, _ = run(bad_k, v, grad)
    assert torch.equal(out[:1200], clean[0][:1200]) and torch.equal(dq[:1200], clean[1][:1200]) and bool(out[1200:].isnan().any())
    bad_grad[600, 1] = math.nan
    _, dq, dk, dv = run(k, v, bad_grad)
    assert torch.equal(dq[:600], clean[1][:600]) and torch.equal(dq[601:], clean[1][601:]) and torch.equal(dq[600, 0], clean[1][600, 0])
    assert torch.equal(dk[601:], clean[2][601:]) and torch.equal(dv[601:], clean[3][601:]) and bool(dv[:601].isnan().any())
