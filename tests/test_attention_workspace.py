"""What a workspace that serves many batches has to hold."""
import pytest

import paper_2508_04405_amd as fq

BATCHES = (1, 2, 3, 5, 8, 16, 17, 31, 33, 64, 65, 100, 128, 129, 257, 600, 1024, 5000)


@pytest.mark.parametrize("heads,kv,D", [(1, 1, 64), (8, 8, 128), (64, 8, 128), (64, 8, 64), (40, 40, 128), (24, 6, 64), (300, 300, 64),
                                        (510, 255, 64), (96, 3, 128)])
def test_one_sequence_of_the_most_rows_needs_most(heads, kv, D):
    size = fq.load().flexq_cache_attention_workspace_bytes
    for most in BATCHES:
        largest = size(most, 1, heads, kv, D)
        assert largest > 0
        for M in (m for m in BATCHES if m <= most):
            for count in BATCHES:
                assert size(M, count, heads, kv, D) <= largest, (most, M, count)
