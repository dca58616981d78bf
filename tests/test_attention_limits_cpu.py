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
