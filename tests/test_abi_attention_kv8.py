"""Workspace of the attention over the 8-bit cache, without a GPU: it follows the work that there is, not the bounds."""
from test_abi import lib  # noqa: F401


def size(lib, sequences, tokens, heads, group, dim, max_q, max_kv):
    return lib.mq_attention_kv8_workspace_size(sequences, tokens, heads, group, dim, max_q, max_kv)


def test_one_long_prompt_among_single_tokens(lib):  # noqa: F811
    """Chunks of some 768 workgroups of 128 columns, each with 131 sums: 52 MB, whatever max_q is."""
    most = 768 * 128 * 131 * 4
    for sequences in (2, 8, 64, 256):
        for heads, group in ((1, 8), (1, 1), (8, 4), (2, 40)):
            for q in (200, 2048, 8191):
                tokens = q + sequences - 1
                items = tokens * group // 128 + sequences
                need = size(lib, sequences, tokens, heads, group, 128, q, 8192)
                assert 0 < need <= most + 8 * items + 16, (sequences, heads, group, q, need)
                # and with max_q left to its default, all rows of Q
                assert 0 < size(lib, sequences, tokens, heads, group, 128, tokens, 8192) <= most + 8 * items + 16


def test_loose_bounds_are_not_refused(lib):  # noqa: F811
    """20 sequences of 1000 queries in all, with bounds far above them (2^24 columns and more, had every sequence max_q)."""
    assert 0 < size(lib, 20, 1000, 1, 8, 128, 1 << 20, 1 << 20) < 100 << 20


def test_many_sequences_under_a_loose_bound(lib):  # noqa: F811
    """Page tables as long as a model's longest context: sums for every 2048 tokens of each of 1024 sequences took 17.6 GB."""
    for sequences in (64, 200, 1024, 5000):
        for heads, group, q in ((8, 4, 1), (8, 8, 8), (1, 8, 1), (32, 1, 1), (2, 16, 4)):
            for dim in (64, 128):
                for max_kv in (8192, 131072, 1 << 20):
                    assert size(lib, sequences, sequences * q, heads, group, dim, q, max_kv) <= 1 << 30
