"""How the products of 8-bit operands are summed, shown by sums of powers of two that are exact."""
import pytest
import torch

from operator_cases import TORCH
from paper_2507_05829_amd import lop

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


def sums_of(pairs, dtype, k=128):
    """One row and output: the sum of x * w over (column, x, w)."""
    x, w = torch.zeros(1, k), torch.zeros(1, k)
    for column, a, b in pairs:
        x[0, column], w[0, column] = a, b
    one = torch.ones(1, -(-k // 128), device="cuda")
    return lop.rowwise_f8(x.to(F8).cuda(), one, w.to(F8).cuda(), one, dtype=TORCH[dtype]).item()


def test_what_the_8_bit_instructions_cut_off():
    """256 * 256 - 256 * 256 + 2^(16 - j): of bf16 results the small product is lost from j = 14 on where it is one of the same eight columns, not
    elsewhere; of fp32 results never. What is kept is cut towards zero."""
    for at, other, small in ((0, 2, 5), (3, 4, 7), (8, 15, 12), (101, 97, 103), (120, 127, 124)):
        for j in range(10, 22):
            half = (16 - j) // 2
            pairs = [(at, 256.0, 256.0), (other, 256.0, -256.0), (small, 2.0 ** half, 2.0 ** (16 - j - half))]
            assert sums_of(pairs, "bf16") == (2.0 ** (16 - j) if j <= 13 else 0.0)
            assert sums_of(pairs, "f32") == 2.0 ** (16 - j)
            elsewhere = pairs[:2] + [((small + 32) % 128, *pairs[2][1:])]
            assert sums_of(elsewhere, "bf16") == 2.0 ** (16 - j)
    for f, kept in ((1.75, 1.5), (-1.75, -1.5), (1.25, 1.0), (-1.25, -1.0)):
        assert sums_of([(0, 256.0, 256.0), (1, 256.0, -256.0), (2, f * 4.0, 4.0)], "bf16") == kept * 16
    # of subnormals the exponent counts (2^-6 * 2^8), of zeros nothing
    for j, kept in ((10, 1), (11, 0)):
        assert sums_of([(0, 2.0 ** -9, 256.0), (1, 2.0 ** -9, -256.0), (2, 2.0 ** (-4 - j + 8), 2.0 ** -5)], "bf16") == kept * 2.0 ** (-1 - j)
    assert sums_of([(0, 0.0, 448.0), (2, 2.0 ** -9, 2.0 ** -9)], "bf16") == 2.0 ** -18
