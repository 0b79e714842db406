"""Inputs and tolerances of the tests of the transformer operators. A rounding to a type is off by half a step, eps / 2 relative to the value."""
import numpy as np
import torch

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
U32 = 2.0 ** -24                                  # half a step of fp32
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def values(rng, shape, dtype, spread=1.0):
    """float32 values that `dtype` holds exactly."""
    t = torch.from_numpy((rng.standard_normal(shape) * spread).astype(np.float32))
    return t.to(TORCH[dtype]).float().numpy()


def product_tolerance(want, size, k, dtype):
    # The products of e4m3 values are exact in fp32. Sums of 128 of them, of the blocks, the two scalings, bias and residual: each
    # addition is off by a step of fp32 at most (the matrix cores may cut rather than round), 2 U32 of what has been added up.
    terms = min(k, 128) + -(-k // 128) + 6
    return HALF[dtype] * np.abs(want) + terms * 2 * U32 * size + 1e-30


def rope_tolerance(want, size, d, dtype):
    # Mean of squares: d / 8 + 3 roundings, half of which the root passes on; root, quotient and two products: 4. The angle: a rounding of up to
    # half a turn (2 pi 2^-26 < 2 U32); cosine and amplitude: 4 + 1; products and sum: 2.
    return HALF[dtype] * np.abs(want) + (d / 16 + 16) * U32 * size + 1e-30


def attention_tolerance(want, size, spread, keys, d, dtype):
    # A score of d products, scaled: off by (d + 4) U32 spread, and so is, relatively, each weight, and their sum; the weights' exponential
    # function 4 U32; sums over the keys; weights rounded for the product with v (bf16) by half a step.
    by_score = (d + 4) * 2 * U32 * spread[..., None]
    relative = 2 * by_score + (2 * keys + 16) * 2 * U32 + (HALF["bf16"] if dtype == "bf16" else 0.0)
    return HALF[dtype] * np.abs(want) + relative * size + 1e-30


def lse_tolerance(want, spread, keys, d):
    return (d + 4) * 2 * U32 * spread.T + (2 * keys + 16) * 2 * U32 + 4 * U32 * np.abs(np.where(np.isfinite(want), want, 0.0))


def assert_near(got, want, tol, what):
    """Equal where `want` is not finite (NaN for NaN), else within tol."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    fine = np.isfinite(want)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want), err_msg=what)
    odd = ~fine & ~np.isnan(want)
    np.testing.assert_array_equal(got[odd], want[odd], err_msg=what)
    off = np.abs(got[fine] - want[fine]) / np.broadcast_to(tol, want.shape)[fine]
    assert off.size == 0 or off.max() <= 1.0, f"{what}: {off.max():.3g} times the tolerance, at {np.argmax(off)}"
