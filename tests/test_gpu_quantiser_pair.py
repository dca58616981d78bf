"""The cache's quantiser and the scores' are one definition, decided by a division here and by a rounded reciprocal there: codes may differ where
32-bit rounding puts an entry next to a tie, and there both levels are as far from it."""
import numpy as np
import pytest

from test_gpu_attention import A, i32, randn, values_of  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("width", [64, 128])
@pytest.mark.parametrize("offset", [0.0, 40.0])
def test_errors_of_the_cache_are_those_the_scores_report(A, bits, width, offset):
    """Squared errors of 8192 rows: an entry next to a tie, within 2^-22 |y / step| steps of it, may change its own by twice that of a step^2."""
    import torch
    from paper_2605_10793_amd import binding
    rows = (randn(3, 8192, 1, width, dtype="f32") * 3 + offset).to(torch.bfloat16)
    cache = A.KVCache.empty(8192 // 256, 1, 256, width, bits)
    table = np.arange(8192 // 256, dtype=np.int32)[None]
    A.append(cache, rows, rows, i32([0, 8192]), i32([0]), i32(table))
    out = torch.zeros(2, dtype=torch.float64, device="cuda:0")
    binding.score_rows_static(rows[:, 0], out, bits=bits, zero_point=True)
    y = rows[:, 0].double()
    step = cache.k_scale[..., 0].reshape(-1, 1).double()
    for which in ("k", "v"):
        value = values_of(cache, which, table[0], 8192)[0][0]
        sse = float((y - value).square().sum())
        # (value = step code + offset as two 32-bit numbers, the scores' as one product; a row's sum in 32 bits)
        slack = float((step.square() * 2.0 ** -20 * (1 + (y / step).abs())).sum()) + 2.0 ** -18 * sse
        assert abs(sse - float(out[0])) <= slack
    assert abs(float(out[1]) - float(y.square().sum())) <= 2.0 ** -18 * float(out[1])
