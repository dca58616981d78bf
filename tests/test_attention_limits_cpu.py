"""Calls at the limits of what the attention operators count, refused or cut before anything is launched."""
from paper_2605_10793_amd import attention as A, binding


def tree_call(columns, sequences, context, bits=8, page_tokens=256):
    """One cache head and one row a sequence; addresses that nothing reads."""
    cache = (0x1000, 0x2000, 0x3000, 0x4000, 4, 1, 64, page_tokens, bits)
    rows = (0x8000, 64, 64, 1)
    return A._TREE.pack(*cache, 0x5000, 0x6000, 0x7000, columns, columns, sequences, *rows, *rows, 0, sequences, context, 0, 0, 1, 0.1)


def test_blocks_of_all_sequences_are_counted_in_31_bits():
    """With what new tokens count for beside their own blocks, and the ends of the last runs: calls of more take a workgroup a sequence and no workspace."""
    lib = binding.load()
    most = (1 << 31) // 512
    for blocks, cut in ((1 << 20, True), (most - 6, True), (most - 5, False), (most - 4, False), (most - 1, False), (most, False)):
        size = lib.conqur_tree_attention_workspace(tree_call(most // 4 + 1, 512, blocks * 64))
        assert (size > 0) == cut, blocks


def chunk_room(bits, tokens, context, sequences=1, max_query=None, heads=32, kv=8, width=128):
    cache = (0x1000, 0x2000, 0x3000 if bits < 16 else 0, 0x4000 if bits < 16 else 0, 1 << 20, kv, width, 64, bits)
    rows = (0x8000, heads * width, width, heads)
    columns = (context + 63) // 64
    return binding.load().conqur_chunk_attention_workspace(A._CHUNK.pack(*cache, 0x5000, 0x6000, 0x7000, columns, columns, sequences, *rows, *rows, 0, 0, 0, tokens, context,
                                                                         0, 0, max_query or tokens // sequences, 0, 0.0, 0.1, 0, 0))


def test_room_that_runs_of_chunk_attention_take():
    """No more than 512 MiB, and none where writing and reading it would take longer than an even share of the work saves; one part a run where there is one sequence."""
    most = 0
    for bits in (16, 8, 4):
        for width in (64, 128):
            for heads, kv in ((32, 8), (64, 1), (8, 8), (40, 40)):
                for tokens in (1, 9, 60, 300, 777, 1024, 2112, 3120, 4160, 8256, 12345, 24600, 60000):
                    for context in (tokens, 16384 + tokens, 1 << 20):
                        for sequences in (1, 2, 3, 16):
                            most = max(most, chunk_room(bits, tokens * sequences, context, sequences, heads=heads, kv=kv, width=width))
    assert 1 << 28 < most <= 1 << 29
    assert chunk_room(16, 4160, 4160) == chunk_room(8, 3120, 3120) == chunk_room(8, 24600, 65536) == 0
    assert chunk_room(8, 777, 30788) == 17 * 192 * 8 * 7 * 130 * 4
    assert chunk_room(16, 1024 * 4, 9024, 4) == 32 * 128 * 8 * 2 * 2 * 130 * 4


def test_runs_of_calls_that_bring_very_different_numbers_of_tokens():
    """The first row tile, which has every sequence, gets the runs that it needs, as far as their room goes; where all bring as many, all tiles get the same."""
    assert chunk_room(16, 640 + 63, 8640, 64, max_query=640) == 20 * 128 * 8 * 2 * 25 * 130 * 4
    assert chunk_room(16, 300 + 7, 8300, 8, max_query=300) == 10 * 128 * 8 * 2 * 30 * 130 * 4
    assert chunk_room(16, 300 * 8, 8300, 8, max_query=300) == 10 * 128 * 8 * 2 * 6 * 130 * 4
