"""Chunk attention of calls whose sequences bring very different numbers of tokens, over contexts that are cut into runs."""
import pytest

from test_gpu_chunk_attention import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits, page, width", [(16, 64, 128), (8, 32, 64), (4, 128, 128)])
@pytest.mark.parametrize("kind, window, cap, biased", [("causal", 0, 0.0, False), ("causal", 900, 0.0, False), ("prefix", 0, 20.0, True)])
def test_a_prompt_among_tokens(bits, page, width, kind, window, cap, biased):
    counts = [1] * 5 + [300] + [1, 0, 2] * 3
    committed = [1500 + (i * 397) % 1500 for i in range(len(counts))]
    check(bits, page, width, committed, counts, 4, 2, kind=kind, window=window, cap=cap, biased=biased, seed=bits, closer=True)


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_one_long_sequence(bits):
    check(bits, 64, 128, [100, 9000, 0, 700, 64], [250, 1, 90, 1, 3], 8, 2, seed=bits, closer=True)
    check(bits, 64, 128, [100, 9000, 0, 700, 64], [250, 1, 90, 1, 3], 8, 2, seed=bits, max_query=200)


def test_two_tiles_of_few_rows():
    check(8, 64, 128, [2000, 3000, 1000, 2500], [7, 1, 1, 1], 8, 2, cap=20.0, closer=True)
    check(8, 16, 128, [2000 + 31 * i for i in range(12)], [7] + [1] * 11, 8, 2, biased=True, closer=True)
