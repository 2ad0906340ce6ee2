"""Sizes that the library's 32-bit arguments cannot hold are refused by the binding."""
import pytest
import torch

import paper_2508_04405_amd as fq
from paper_2508_04405_amd.binding import _rows


def rows(stride, count=2):
    return torch.empty_strided((count, 1024), (stride, 1), dtype=torch.float16, device="meta")


def test_strides_past_32_bits():
    """2^32 + 1024 would be taken for 1024."""
    for stride in (2**31, 2**32 + 1024, 2**40 + 1024):
        with pytest.raises(fq.FlexQError):
            _rows(rows(stride), 2, 1024, -1)
    assert _rows(rows(2**31 - 8), 2, 1024, -1) == 2**31 - 8
    assert _rows(rows(2**32 + 1024, 1), 1, 1024, -1) == 1024          # (one row has no next one)


@pytest.mark.gpu
def test_a_table_past_32_bits():
    i32 = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")
    table = torch.empty((1, 2**32 + 4), dtype=torch.int32, device="cuda")     # would be taken for four pages
    with pytest.raises(fq.FlexQError):
        fq.Sequences(i32(2), i32(1), table)
