"""Head norms of values whose squares fp32 does not hold."""
import numpy as np
import pytest
import torch

from operator_cases import TORCH, assert_near, rope_tolerance, values
from oracle import transformer as plain
from paper_2507_05829_amd import lop

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 72, 128, 256])
@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-6, 1.0])
def test_values_of_all_sizes(eps, d, dtype):
    """A head for each power of two from 2^-110 to 2^120, ordinary heads between them; no rotation."""
    rng = np.random.default_rng(d)
    powers = np.arange(-110, 121, 5)
    x = values(rng, (3, len(powers), d), dtype) * np.exp2(powers).astype(np.float32)[None, :, None]
    x[1] = values(rng, (len(powers), d), dtype)
    w = (1 + 0.1 * rng.standard_normal(d)).astype(np.float32)
    t = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    got, _ = lop.head_norm_rope(t(x).to(TORCH[dtype]), None, None, None, q_weight=t(w), eps=eps)
    want, size = plain.norm_rope(x, None, None, w, float(np.float32(eps)), False, 1.0)
    # (beside the roundings that rope_tolerance counts: values below fp32's normal ones, of results of 2^-126 and less)
    assert_near(got.float().cpu().numpy(), want, rope_tolerance(want, size, d, dtype) + 2.0 ** -126, "norms")


def test_zeros_infinities_and_nans():
    x = torch.ones(4, 2, 64, device="cuda")
    x[0] = 0.0
    x[1, 0, 5], x[2, 1, 63] = float("inf"), float("nan")
    w = torch.ones(64, device="cuda")
    for eps in (0.0, 1e-6):
        got, _ = lop.head_norm_rope(x, None, None, None, q_weight=w, eps=eps)
        assert got[0].isnan().all() if eps == 0 else (got[0] == 0).all()
        assert got[1, 0, 5].isnan() and (got[1, 0, :5] == 0).all() and got[2, 1].isnan().all()
        assert torch.allclose(got[3], torch.ones_like(got[3]), rtol=2e-6, atol=0) and torch.equal(got[1, 1], got[3, 1]) and torch.equal(got[2, 0], got[3, 0])
