"""A row of attention depends on its own query and the keys and values it sees: bit for bit, whatever stands beside it, as long as
the keys are cut alike."""
import numpy as np
import pytest
import torch

from operator_cases import TORCH, values
from paper_2507_05829_amd import lop
from test_operators_gpu import attend, check_attention, packed

pytestmark = pytest.mark.gpu


def same(got, want, rows=slice(None)):
    for a, b in zip(got, want):
        if a.ndim == 2:                     # logarithms: (heads, rows)
            a, b = a.T, b.T
        np.testing.assert_array_equal(a[rows].view(np.uint32), b[rows].view(np.uint32))


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("f32", 128), ("f32", 256), ("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("grow", [0.0, 0.4])
def test_a_band_is_the_whole_calls(dtype, d, grow):
    """grow: keys become longer from token to token, so that maxima grow now in one row, now in another."""
    rng = np.random.default_rng(d)
    q, k, v, o, b, e = packed(rng, [(50, 50), (190, 400), (3, 9)], 4, 2, d, dtype)
    k = torch.from_numpy((k * (1 + grow * np.arange(len(k)) ** 0.5)[:, None, None]).astype(np.float32)).to(TORCH[dtype]).float().numpy()
    whole = attend(q, k, v, o, b, e, dtype, max_keys=1)
    for lo, hi in ((0, 1), (17, 90), (64, 243), (128, 129)):
        part = attend(q, k, v, o, b, e, dtype, max_keys=1, rows=(lo, hi))
        same(part, whole, slice(lo, hi))


@pytest.mark.parametrize("max_keys", [1, 5000])
@pytest.mark.parametrize("dtype,d", [("f32", 64), ("f32", 128), ("f32", 256), ("bf16", 64), ("bf16", 128)])
def test_rows_beside_it_do_not_change_a_row(dtype, d, max_keys):
    """Other queries (some of them NaN or infinite, others with scores that grow all the time) in the rows beside it."""
    rng = np.random.default_rng(d + 1)
    q, k, v, o, b, e = packed(rng, [(40, 600), (30, 64)], 4, 2, d, dtype)
    k = torch.from_numpy((k * (1 + np.arange(len(k)) / 50.0)[:, None, None]).astype(np.float32)).to(TORCH[dtype]).float().numpy()
    before = attend(q, k, v, o, b, e, dtype, max_keys=max_keys)
    kept = np.arange(70) % 3 == 0
    for what in (7.0, 0.0, np.nan, np.inf, 1e30):
        other = q.copy()
        other[~kept] = values(rng, other[~kept].shape, dtype) * np.float32(7.0) if what == 7.0 else what
        same(attend(other, k, v, o, b, e, dtype, max_keys=max_keys), before, kept)


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("f32", 128), ("f32", 256), ("bf16", 64), ("bf16", 128)])
def test_later_tokens_do_not_change_a_row(dtype, d):
    """The first 100 tokens of a prompt are what they are without the others."""
    rng = np.random.default_rng(d + 2)
    q, k, v, o, b, e = packed(rng, [(300, 300)], 4, 2, d, dtype)
    k[100:] *= 8.0
    short = attend(q[:100], k[:100], v[:100], [0, 100], [0], [100], dtype, max_keys=1)
    long = attend(q, k, v, o, b, e, dtype, max_keys=1)
    same((long[0][:100], long[1][:, :100]), short)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("max_keys", [1, 5000])
@pytest.mark.parametrize("d", [8, 72, 96, 128, 136, 256])
def test_hidden_values_of_all_head_sizes(d, max_keys, dtype):
    """Some rows of a workgroup go through their keys again, others not: later tokens' values are NaN or infinite, one key of the second sequence has scores
    far from the others', one value of it is infinite, and the third sequence sees its last tile partly."""
    rng = np.random.default_rng(d + 3)
    q, k, v, o, b, e = packed(rng, [(70, 70), (9, 300), (130, 190)], 6, 2, d, dtype, room=320)
    v[b[0] + 40:e[0], 0, :3] = np.nan
    v[b[0] + 60:e[0], 1, d - 1] = np.inf
    k[b[1] + 17] *= np.float32(2.0 ** 60)
    v[b[1] + 299, 1] = -np.inf
    v[b[2] + 150:e[2]:7] = np.nan
    check_attention(attend(q, k, v, o, b, e, dtype, max_keys=max_keys), q, k, v, o, b, e, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("max_keys", [1, 5000])
@pytest.mark.parametrize("d", [8, 40, 72, 120, 128, 200])
def test_what_lies_between_rows_and_heads_is_not_read(d, max_keys, dtype):
    """Heads of d values in places for more, NaNs behind them; and an output in such places, which keeps what is behind them."""
    rng = np.random.default_rng(d + 4)
    q, k, v, o, b, e = packed(rng, [(20, 150), (3, 40)], 4, 2, d, dtype)
    plain_out, _ = attend(q, k, v, o, b, e, dtype, max_keys=max_keys)
    dt, room = TORCH[dtype], d + 24

    def inside(a):
        t = torch.full((a.shape[0], a.shape[1], room), float("nan"), dtype=dt, device="cuda")
        t[..., :d] = torch.from_numpy(a).cuda().to(dt)
        return t[..., :d]

    out = inside(np.zeros_like(q))
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    lop.attention(inside(q), inside(k), inside(v), i32(o), i32(b), i32(e), d ** -0.5, max_keys=max_keys, out=out)
    np.testing.assert_array_equal(out.float().cpu().numpy(), plain_out)
    assert out.as_strided((q.shape[0], 4, 24), (4 * room, room, 1), d).isnan().all()
