"""Outputs of the transformer operators whose rows, heads or scales would share memory are refused, on the host; what lies apart in
an unusual order is not. No kernel is launched: the calls that pass these checks are such that a later one refuses them."""
import itertools

import pytest

from paper_2507_05829_amd import lop
from test_operators_host import ARG, UNS, attention_op, quantize_op, refused, rope_op

STRIDES = (64, 72, 96, 104, 128, 136, 192, 200, 264, 320, 328, 512, 1024)


def overlap(extents, strides, inner):
    """Whether two of the places that the strides lead to are less than `inner` elements apart, by trying all."""
    at = sorted(sum(i * s for i, s in zip(where, strides)) for where in itertools.product(*(range(n) for n in extents)))
    return any(b - a < inner for a, b in zip(at, at[1:]))


@pytest.mark.parametrize("rows,heads", [(1, 4), (4, 1), (2, 2), (3, 4), (7, 2), (5, 3), (6, 6)])
def test_attention_outputs(rows, heads):
    """(Keys too far apart are what is refused last.)"""
    for token, head in itertools.product(STRIDES, STRIDES):
        op = attention_op()
        op.rows_q, op.heads_q, op.heads_k, op.k_token = rows, heads, 1, 1 << 24
        refused(lop.lop_attention, op, (0, rows), ARG if overlap((rows, heads), (token, head), 64) else UNS, out_token=token, out_head=head)


def test_attention_outputs_far_apart_and_of_many_rows():
    n = 1 << 16
    for code, rows, heads, token, head in ((UNS, n, 512, 64, 64 * n), (ARG, n, 512, 64, 64 * n - 64), (UNS, n, 512, 512 * 64, 64), (ARG, n, 512, 511 * 64, 64),
                                           (UNS, n, 2, 1 << 59, 1 << 58), (UNS, n, 2, 1 << 58, 1 << 59 | 64), (ARG, n, 3, 1 << 58, 1 << 58)):
        op = attention_op()
        op.rows_q, op.heads_q, op.heads_k, op.k_token = rows, heads, 1, 1 << 24
        refused(lop.lop_attention, op, (0, 5), code, out_token=token, out_head=head)


@pytest.mark.parametrize("change", [dict(q_out_token=64), dict(q_out_token=128), dict(k_out_token=64), dict(q_out_token=192), dict(q_out_head=256), dict(k_out_head=128), dict(q_out_head=64 * 48),
                                    dict(k_out_token=96, k_out_head=64)])
def test_rope_outputs(change):
    refused(lop.lop_head_norm_rope, rope_op(), (0, 9), ARG, **change)


@pytest.mark.parametrize("block_rows,change", [(1, dict(scale_row=0)), (1, dict(scale_col=0)), (1, dict(scale_row=0, scale_col=0)), (1, dict(scale_row=1, scale_col=199)), (1, dict(scale_row=2, scale_col=2)),
                                               (1, dict(scale_row=1, scale_col=1)), (128, dict(scale_row=0, scale_col=1)), (128, dict(scale_row=1, scale_col=1))])
def test_scales(block_rows, change):
    refused(lop.lop_quantize_blocks, quantize_op(), (0, 128), ARG, block_rows=block_rows, **change)


def test_scales_of_one_column_or_row_may_have_any_stride():
    """(More workgroups than a launch takes are what is refused last.)"""
    for code, change in ((UNS, dict(k=128, scale_row=1, scale_col=0)), (ARG, dict(k=128, scale_row=0, scale_col=1)), (UNS, dict(k=1 << 20, scale_row=1 << 20, scale_col=1)),
                         (ARG, dict(k=1 << 20, scale_row=1, scale_col=(1 << 31) - 2)), (UNS, dict(k=1 << 20, scale_row=1, scale_col=(1 << 31) - 1)), (UNS, dict(k=1 << 20, scale_row=1 << 13, scale_col=1))):
        op = quantize_op()
        op.m, op.dtype, op.x_stride, op.q_stride = (1 << 31) - 1, lop.LOP_F32, 1 << 20, 1 << 20
        refused(lop.lop_quantize_blocks, op, (0, op.m), code, **change)
