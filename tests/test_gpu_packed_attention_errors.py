"""Attention's errors and its gradients', squared and summed, are those of two roundings to bf16, and dq's those of one.

A rounding to 8 bits of a number whose mantissa m lies anywhere in [1, 2), by its logarithm, is off by 2^-7 / sqrt(12) / m relative, squared and averaged over m
2^-14 / 12 * 3 / (8 ln 2), the root of which is 0.00166.  A result is rounded once, and is a sum over factors that are rounded, each by itself (weights for out and
dv, du for dk): as the terms of such a sum are of either sign, as good as at random, it is off by no more than one rounding of what it is.  Together sqrt(2) times
0.00166.  dq's factors are in two parts, and what the rounded weights in lse and the rounded result in D make of it is taken out, so that its own rounding is left.
A tenth is added for 32-bit sums and for what is left of D and lse.
"""
import pytest
import torch

from attention_reference import attend, seen_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ONE = 1.1 * (2.0 ** -14 / 12 * 3 / (8 * 0.6931471805599453)) ** 0.5
TWO = 2 ** 0.5 * ONE


@pytest.mark.parametrize("width", [64, 128])
@pytest.mark.parametrize("n, heads, kv, cap, biased", [(700, 8, 2, 0.0, False), (700, 8, 2, 20.0, False), (700, 8, 2, 0.0, True), (2300, 2, 1, 0.0, False)])
def test_errors_are_those_of_roundings(width, n, heads, kv, cap, biased):
    """Many rows a workgroup, and few whose keys several workgroups share."""
    from paper_2605_10793_amd import attention as A
    g = torch.Generator().manual_seed(n + width)
    q, k, v, grad = (torch.randn(n, h, width, generator=g).to(torch.bfloat16) for h in (heads, kv, kv, heads))
    slopes = torch.exp2(-8 * (1 + torch.arange(heads, dtype=torch.float32)) / heads) if biased else None
    start = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    options = dict(cap=cap, slopes=None if slopes is None else slopes.to(DEV))
    on = [x.to(DEV) for x in (q, k, v, grad)]
    out, lse = A.attention(*on[:3], start, lse=True, **options)
    got = dict(zip(("out", "dq", "dk", "dv"), (out, *A.attention_backward(*on[:3], out, lse, on[3], start, **options))))
    want = attend(q, k, v, seen_of(n, None, None, 0), torch.arange(n), width ** -0.5, cap, slopes, grad=grad)
    off = {name: float((x.cpu().double() - want[name]).norm() / want[name].norm()) for name, x in got.items()}
    assert max(off["out"], off["dk"], off["dv"]) <= TWO and off["dq"] <= ONE, off
