"""Attention of a packed sequence of more tokens than 24 bits count."""
import pytest
import torch

from attention_reference import attend, close

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_distances_behind_2_to_the_24(cap):
    """A window and a bias by distance: results and gradients of the last tokens, whose numbers 32-bit floats do not hold."""
    from paper_2605_10793_amd import attention as A
    n, window, last, width = (1 << 24) + 301, 40, 200, 32
    g = torch.Generator(device=DEV).manual_seed(int(cap))
    q, k, v, grad = (torch.randn(n, 1, width, device=DEV, dtype=torch.bfloat16, generator=g) for _ in range(4))
    slopes, start = torch.tensor([0.7]), torch.tensor([0, n], dtype=torch.int32, device=DEV)
    options = dict(window=window, cap=cap, slopes=slopes.to(DEV))
    out, lse = A.attention(q, k, v, start, lse=True, **options)
    grads = A.attention_backward(q, k, v, out, lse, grad, start, **options)
    # The last rows and the keys that they see, which no others see but for the first window of them.
    part = [x[n - last - window:].cpu() for x in (q, k, v, grad)]
    place, j = torch.arange(last + window)[:, None], torch.arange(last + window)[None]
    want = attend(*part[:3], (j <= place) & (j > place - window), place[:, 0], width ** -0.5, cap, slopes, grad=part[3])
    for name, x in zip(("out", "dq", "dk", "dv"), (out, *grads)):
        close(x[n - last:], want[name][window:], want[name + "_tol"][window:], name)
