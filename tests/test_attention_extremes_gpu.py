"""Attention of scores and values near the ends of fp32's range, on the GPU."""
import numpy as np
import pytest
import torch

from operator_cases import HALF, U32, attention_tolerance, lse_tolerance, values
from oracle import transformer as plain
from test_operators_gpu import attend

pytestmark = pytest.mark.gpu


def near(got, want, d, dtype, keys, size=None):
    """Where the weights of a row are exactly known: weights and output rounded to bf16, exponential function (4 U32), sums of the weights and of
    their products with v, a quotient and a product for each tile of at least 32 keys."""
    size = np.abs(want) if size is None else size
    roundings = 2 * HALF["bf16"] if dtype == "bf16" else HALF["f32"]
    tol = roundings * size + (2 * keys + 4 * (keys // 32 + 1) + 16) * 2 * U32 * size + 1e-37
    off = np.abs(np.asarray(got, np.float64) - want)
    assert np.isfinite(got).all() and (off <= tol).all(), f"{np.nanmax(off / tol):.3g} times the tolerance"


@pytest.mark.parametrize("size", [1e10, 1e20, 2.4e24, 1e30, 1e37])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
@pytest.mark.parametrize("d,dtype", [(64, "f32"), (96, "f32"), (128, "f32"), (256, "f32"), (64, "bf16"), (256, "bf16")])
def test_scores_far_from_zero(d, dtype, sign, size):
    """Scores of +-size, by far the same key for every row: a causal row sees one key more than the row before it, all of them with the
    same score, so that its output is the mean of the values."""
    rng = np.random.default_rng(d)
    n = 70
    a = torch.tensor((size / d) ** 0.5).to(torch.bfloat16).float().item()
    q, k = np.full((n, 2, d), a, np.float32), np.full((n, 1, d), sign * a, np.float32)
    v = values(rng, (n, 1, d), dtype)
    out, lse = attend(q, k, v, [0, n], [0], [n], dtype, scale=0.125)
    count = np.arange(1, n + 1)[:, None, None]
    near(out, np.broadcast_to(np.cumsum(v.astype(np.float64), 0) / count, out.shape), d, dtype, n,
         np.broadcast_to(np.cumsum(np.abs(v.astype(np.float64)), 0) / count, out.shape))
    score = 0.125 * sign * float(a) * float(a) * d
    want = score + np.log(np.arange(1, n + 1))
    spread = np.full((n, 2), abs(score))
    assert (np.abs(lse - want) <= lse_tolerance(np.broadcast_to(want, (2, n)), spread, n, d)).all()


@pytest.mark.parametrize("d,dtype", [(64, "f32"), (128, "f32"), (256, "f32"), (128, "bf16")])
def test_scores_far_from_zero_of_cut_keys(d, dtype):
    """The same in parts of the keys, some of which a row does not see, and one key of a score closer to zero, whose value is the result."""
    rng = np.random.default_rng(d + 1)
    n, seqs = 900, 3
    a = torch.tensor((3e25 / d) ** 0.5).to(torch.bfloat16).float().item()
    q, k = np.full((2 * seqs, 2, d), a, np.float32), np.full((seqs * n, 1, d), -a, np.float32)
    k[n + 500] *= 0.5
    v = values(rng, (seqs * n, 1, d), dtype)
    begin, end = [0, n, 2 * n], [n, 2 * n, 2 * n + 40]
    out, _ = attend(q, k, v, [0, 2, 4, 6], begin, end, dtype, scale=0.125, max_keys=n)
    for i, sees in ((0, n - 1), (1, n), (4, 39), (5, 40)):
        seen = v[begin[i // 2]:begin[i // 2] + sees, 0].astype(np.float64)
        near(out[i], np.broadcast_to(seen.mean(0), (2, d)), d, dtype, n, np.broadcast_to(np.abs(seen).mean(0), (2, d)))
    near(out[2:4], np.broadcast_to(v[n + 500], (2, 2, d)).astype(np.float64), d, dtype, 1)


@pytest.mark.parametrize("max_keys", [1, 5000])
@pytest.mark.parametrize("scale", [0.125, 2.0 ** -80])
def test_scores_whose_terms_cancel(scale, max_keys):
    """Every even key's score is 0, a sum of terms of -2^84 and 2^84 whose order the kernel chooses; every odd key's is -2^86 (where
    the scale is small a weight of e^-64 beside 1). One row sees one odd key only."""
    rng = np.random.default_rng(3)
    n, d = 160, 64
    q = np.full((3, 1, d), 2.0 ** 42, np.float32)
    k = np.full((n, 1, d), 2.0 ** 38, np.float32)
    k[:, :, ::2] *= -1.0
    k[1::2] = -(2.0 ** 38)
    v = values(rng, (n, 1, d), "f32")
    out, _ = attend(q, k, v, [0, 2, 3], [0, 1], [n, 2], "f32", scale=scale, max_keys=max_keys)
    want, _, size, _ = plain.attention(q, k, v, [0, 2, 3], [0, 1], [n, 2], scale, True)
    near(out, want, d, "f32", n, size)


@pytest.mark.parametrize("scale", [2.0 ** -81, 2.0 ** -90])
def test_far_scores_of_a_small_scale(scale):
    """Scores from -2^82 to 2^82 whose scaled differences are of the order of one."""
    rng = np.random.default_rng(4)
    n, d = 130, 64
    q = np.full((2, 1, d), 2.0 ** 40, np.float32)
    k = np.broadcast_to(np.round(rng.uniform(-64, 64, (n, 1, 1))) * np.float32(2.0 ** 30), (n, 1, d)).astype(np.float32)
    v = values(rng, (n, 1, d), "f32")
    out, _ = attend(q, k, v, [0, 2], [0], [n], "f32", scale=scale)
    want, _, size, spread = plain.attention(q, k, v, [0, 2], [0], [n], scale, True)
    # scores are exact (sums of up to 64 times a whole number below 2^7 times a power of two); scaled and by the logarithm of 2: 2 roundings each,
    # in the difference of two of up to `spread`: relative in the weights
    near(out, want, d, "f32", n, size * (1 + 8 * U32 * spread[..., None] / (2 * n * 2 * U32)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("max_keys", [1, 5000])
@pytest.mark.parametrize("size", [2.0 ** 110, 2.0 ** 116, 2.0 ** 127])
def test_values_near_the_end_of_the_range(size, max_keys, dtype):
    """Scores that grow a little from key to key, so that the weights relative to those of the first keys are large, and values whose weighted mean is
    finite while their sums are not."""
    rng = np.random.default_rng(5)
    n, d = 600, 64
    q = np.zeros((3, 2, d), np.float32)
    q[..., 0] = 1.0
    k = np.zeros((n, 1, d), np.float32)
    k[:, 0, 0] = np.floor(np.arange(n) / 64.0) * 2.0
    v = (values(rng, (n, 1, d), dtype).clip(0.25, 1.0) * np.float32(size)).astype(np.float32)
    out, _ = attend(q, k, v, [0, 1, 3], [0, 0], [n, 200], dtype, scale=1.0, max_keys=max_keys)
    want, _, mean, spread = plain.attention(q, k, v, [0, 1, 3], [0, 0], [n, 200], 1.0, True)
    near(out, want, d, dtype, n, mean * (1 + 8 * U32 * spread[..., None] / (2 * n * 2 * U32)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("max_keys", [1, 5000])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
def test_scores_past_the_range_show(sign, max_keys, dtype):
    """Rows of which every score is +-6.4e40 are NaN; where one key's score is 0 and the others' -6.4e40, its value is the result."""
    rng = np.random.default_rng(6)
    n, d = 200, 64
    q, k = np.full((2, 1, d), 2.0 ** 66, np.float32), np.full((2 * n, 1, d), sign * 2.0 ** 63, np.float32)
    k[n + 50] = 0.0
    v = values(rng, (2 * n, 1, d), dtype)
    out, _ = attend(q, k, v, [0, 1, 2], [0, n], [n, 2 * n], dtype, scale=0.125, max_keys=max_keys)
    assert np.isnan(out[0]).all()
    if sign > 0:
        assert np.isnan(out[1]).all()
    else:
        near(out[1], v[n + 50].astype(np.float64), d, dtype, 1)


@pytest.mark.parametrize("max_keys", [1, 5000])
@pytest.mark.parametrize("power", [80, 110, 120])
def test_operands_far_apart(power, max_keys):
    """Queries of about 2^power against keys of about 2^-power and values of 2^power / 4: ordinary scores of operands that are anything but."""
    rng = np.random.default_rng(7)
    q, k, v = (values(rng, (n, 1, 64), "f32") for n in (4, 300, 300))
    tall = [np.float32(2.0 ** power) * q, np.float32(2.0 ** -power) * k, np.float32(2.0 ** (power - 2)) * v]
    o, b, e = [0, 3, 4], [0, 10], [300, 11]
    out, lse = attend(*tall, o, b, e, "f32", max_keys=max_keys)
    want, want_lse, size, spread = plain.attention(*tall, o, b, e, 0.125, True)
    tol = attention_tolerance(want, size, spread, 300, 64, "f32")
    assert np.isfinite(out).all() and (np.abs(out - want) <= tol).all()
    assert (np.abs(lse - want_lse) <= lse_tolerance(want_lse, spread, 300, 64)).all()
