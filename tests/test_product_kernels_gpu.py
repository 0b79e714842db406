"""Every kernel of the product of 8-bit operands against 64 bits (formed on the GPU by a library product of doubles), all outputs
one by one. That each product is run by the kernel it is for is a host test."""
import pytest
import torch

from operator_cases import HALF, TORCH, U32
from paper_2507_05829_amd import lop
from product_cases import FLAT

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


def operands(gen, rows, k, scale_rows):
    """Values of all sizes, scales that differ from block to block by a factor of up to four."""
    v = (torch.randn(rows, k, device="cuda", generator=gen) * 60).clamp_(-448, 448).to(F8)
    return v, torch.exp2(torch.rand(scale_rows, -(-k // 128), device="cuda", generator=gen) * 2 - 9)


def in_64_bits(x, xs, w, ws, dtype):
    """(sums of products, what they may be off by before the rounding of the result).

    Each addition in fp32 is off by a step of what has been added up, as product_tolerance in operator_cases.py counts. bf16 results: the 8-bit instructions cut the products of each
    eight neighbouring columns off at 2^-13 of 2^E, E the largest sum of two operands' exponents among them, where subnormal operands have
    that of 2^-6 and zeros none (test_product_rounding_gpu.py). 2^E is at most |x'| |w'| of that column, with x' and w' the operands raised to
    2^-6, of which the seven others are off by less than 2^-13 each: 7 * 2^-13 times the sum of |x'| |w'| over the columns bounds it for all eights together."""
    k, n = x.shape[1], w.shape[0]
    xs = xs.double().repeat_interleave(128, 1)[:, :k]
    ws = ws.double().repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :k]
    a, b = x.double(), w.double()
    off = ((a.abs() * xs) @ (b.abs() * ws).t().contiguous()) * ((min(k, 128) + -(-k // 128) + 6) * 2 * U32)
    if dtype == "bf16":
        raised = lambda t: torch.where(t == 0, 0.0, t.abs().clamp(min=2.0 ** -6))  # noqa: E731
        off += ((raised(a) * xs) @ (raised(b) * ws).t().contiguous()) * (7 * 2.0 ** -13)
    return (a * xs) @ (b * ws).t().contiguous(), off


def check(got, want, off, dtype, what, terms=0.0):
    """terms: magnitudes of what was added in fp32 afterwards: up to 8 steps more."""
    tol = HALF[dtype] * want.abs() + off + 16 * U32 * terms + 1e-30
    off = ((got.double() - want).abs() / tol).max().item()
    assert off <= 1.0, f"{what}: {off:.3g} times the tolerance"


def wider(t, before, behind):
    """The same values inside a buffer with more columns, NaNs."""
    buf = torch.full((t.shape[0], before + t.shape[1] + behind), float("nan"), device="cuda").to(t.dtype)
    buf[:, before:before + t.shape[1]] = t
    return buf[:, before:before + t.shape[1]]


@pytest.mark.parametrize("kernel,dtype,m,k,n", FLAT)
def test_product_kernel(kernel, dtype, m, k, n):
    """A band of m rows out of m + 7: alone; with bias, activation and residual; and with results that begin anywhere, the residual in place, operands in wider
    buffers and scales in the other order. Twice each: the same bits."""
    gen = torch.Generator(device="cuda").manual_seed(m * 31 + k * 7 + n)
    dt, lo, hi = TORCH[dtype], 3, m + 3
    x, xs = operands(gen, m + 7, k, m + 7)
    w, ws = operands(gen, n, k, -(-n // 128))
    bias = torch.randn(n, device="cuda", generator=gen)
    res = torch.randn(m + 7, n, device="cuda", generator=gen).to(dt)
    want, off = in_64_bits(x[lo:hi], xs[lo:hi], w, ws, dtype)

    def outside_is(y, before):
        assert torch.equal(y[:lo], before[:lo]) and torch.equal(y[hi:], before[hi:])

    def twice(call):
        y = call()
        assert torch.equal(call(), y), "two runs differ"
        return y

    # alone, aligned where n is a multiple of 8
    sevens = torch.full((m + 7, n), 7.0, dtype=dt, device="cuda")
    xs_t = xs.t().contiguous().t()
    y = twice(lambda: lop.rowwise_f8(x, xs_t, w, ws, y=sevens.clone(), rows=(lo, hi)))
    outside_is(y, sevens)
    check(y[lo:hi], want, off, dtype, "alone")

    added = want + bias.double() + res[lo:hi].double()
    terms = want.abs() + bias.double().abs() + res[lo:hi].double().abs()
    y = twice(lambda: lop.rowwise_f8(x, xs_t, w, ws, bias=bias, act="relu", residual=res, y=sevens.clone(), rows=(lo, hi)))
    outside_is(y, sevens)
    check(y[lo:hi], added.clamp(min=0), off, dtype, "with bias, residual and relu", terms)

    x2, w2, ws_t = wider(x, 32, 48), wider(w, 16, 16), ws.t().contiguous().t()

    def in_place():
        buf = torch.full((m + 7, n + 9), 7.0, dtype=dt, device="cuda")
        y = buf[:, 3:3 + n]
        y.copy_(res)
        lop.rowwise_f8(x2, xs, w2, ws_t, bias=bias, act="relu6", residual=y, y=y, rows=(lo, hi))
        assert (buf[:, :3] == 7).all() and (buf[:, 3 + n:] == 7).all()
        return y.clone()

    y = twice(in_place)
    outside_is(y, res)
    check(y[lo:hi], added.clamp(0, 6), off, dtype, "in place, anywhere", terms)


def test_odd_values_stay_in_their_rows_and_columns():
    """Of the kernels with tiles in LDS: NaNs and an infinite scale show in their own rows and columns and nowhere else."""
    for kernel, dtype, m, k, n in [c for c in FLAT if "few" not in c[0]][::3]:
        gen = torch.Generator(device="cuda").manual_seed(m)
        x, xs = operands(gen, m, k, m)
        w, ws = operands(gen, n, k, -(-n // 128))
        want, off = in_64_bits(x, xs, w, ws, dtype)
        x.view(torch.uint8)[3, k - 1] = 0x7f
        xs[m - 2, 0] = float("inf")
        w.view(torch.uint8)[n - 1, 0] = 0x7f
        y = lop.rowwise_f8(x, xs, w, ws, act="relu", dtype=TORCH[dtype])
        assert y[3].isnan().all() and y[:, n - 1].isnan().all()
        clean = torch.ones(m, dtype=torch.bool, device="cuda")
        clean[3] = clean[m - 2] = False
        check(y[clean, :n - 1], want[clean, :n - 1].clamp(min=0), off[clean, :n - 1], dtype, f"{m} x {k} to {n}")
