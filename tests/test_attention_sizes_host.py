"""Sizes of attention at the end of 32 bits, without a GPU. (Keys too far apart are what is refused last.)"""
import pytest

from paper_2507_05829_amd import lop
from test_operators_host import UNS, attention_op, refused


@pytest.mark.parametrize("rows_k", [(1 << 31) - 64, (1 << 31) - 33, (1 << 31) - 1])
def test_keys_whose_last_tile_ends_past_32_bits_are_refused(rows_k):
    op = attention_op()
    refused(lop.lop_attention, op, (0, 9), UNS, rows_k=rows_k)
    with pytest.raises(lop.LopError) as e:
        lop.lop_attention_workspace(op, (0, 9))
    assert e.value.code == UNS


def test_the_longest_keys_are_not():
    op = attention_op()
    op.rows_k = op.max_keys = (1 << 31) - 65
    assert lop.lop_attention_workspace(op, (0, 9)) > 0
    refused(lop.lop_attention, op, (0, 9), UNS, k_token=1 << 24)
