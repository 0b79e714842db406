"""The transformer operators without a GPU: what the library refuses, sizes of workspaces, and the pins of their plain 64-bit
forms against third-party routines and closed forms. No kernel is launched."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import transformer as plain
from paper_2507_05829_amd import lop

A = 0x1000            # an address that is never touched
BAND, ARG, UNS, SHAPE = lop.LOP_ERR_BAND_RANGE, lop.LOP_ERR_INVALID_ARG, lop.LOP_ERR_UNSUPPORTED, lop.LOP_ERR_SHAPE


def refused(call, op, rows, code, **change):
    for name, v in change.items():
        assert hasattr(op, name)
        setattr(op, name, v)
    with pytest.raises(lop.LopError) as e:
        call(op, rows)
    assert e.value.code == code, (change, e.value.code)


def quantize_op():
    return lop.lop_quantize_t(200, 256, lop.LOP_BF16, 1, A, 256, A, 256, A, 1, 200)


@pytest.mark.parametrize("code,rows,change", [
    (ARG, (0, 9), dict(x=None)), (ARG, (0, 9), dict(q=None)), (ARG, (0, 9), dict(scale=None)), (ARG, (0, 9), dict(x=A + 8)), (ARG, (0, 9), dict(q=A + 4)),
    (ARG, (0, 9), dict(scale=A + 2)), (ARG, (0, 9), dict(x_stride=260)), (ARG, (0, 9), dict(q_stride=-256)), (ARG, (0, 9), dict(q_stride=264)), (ARG, (0, 9), dict(q_stride=240)), (ARG, (0, 9), dict(scale_row=-1)),
    (ARG, (0, 0), dict(m=-1)), (ARG, (0, 0), dict(k=0)), (UNS, (0, 9), dict(k=250)), (UNS, (0, 9), dict(dtype=2)), (UNS, (0, 9), dict(block_rows=64)),
    (BAND, (-1, 9), {}), (BAND, (9, 8), {}), (BAND, (0, 201), {}), (BAND, (64, 200), dict(block_rows=128)), (BAND, (0, 100), dict(block_rows=128))])
def test_quantize_refuses(code, rows, change):
    refused(lop.lop_quantize_blocks, quantize_op(), rows, code, **change)


def product_op():
    return lop.lop_rowwise_f8_t(100, 60, 256, lop.LOP_BF16, 0, A, 256, A, 1, 100, A, 256, A, 2, 1, None, None, 0, A, 60)


@pytest.mark.parametrize("code,rows,change", [
    (ARG, (0, 9), dict(x=None)), (ARG, (0, 9), dict(w=None)), (ARG, (0, 9), dict(x_scale=None)), (ARG, (0, 9), dict(w_scale=None)), (ARG, (0, 9), dict(y=None)),
    (ARG, (0, 9), dict(x=A + 8)), (ARG, (0, 9), dict(w=A + 1)), (ARG, (0, 9), dict(y=A + 1)), (ARG, (0, 9), dict(residual=A + 1, residual_stride=60)),
    (ARG, (0, 9), dict(bias=A + 2)), (ARG, (0, 9), dict(x_scale=A + 1)), (ARG, (0, 9), dict(x_stride=257)), (ARG, (0, 9), dict(w_stride=-16)),
    (ARG, (0, 9), dict(y_stride=-60)), (ARG, (0, 9), dict(y_stride=59)), (ARG, (0, 9), dict(x_scale_row=-1)), (ARG, (0, 9), dict(w_scale_col=-1)), (ARG, (0, 9), dict(n=0)), (ARG, (0, 0), dict(k=0)),
    (UNS, (0, 9), dict(k=100)), (UNS, (0, 9), dict(dtype=7)), (UNS, (0, 9), dict(act=3)), (UNS, (0, 9), dict(act=-1)), (UNS, (0, 9), dict(x_stride=1 << 24)),
    (UNS, (0, 9), dict(w_stride=1 << 24)), (UNS, (0, 9), dict(x_scale_row=1 << 24)), (UNS, (0, 9), dict(k=1 << 24)), (BAND, (0, 101), {}), (BAND, (5, 4), {}), (BAND, (-2, 4), {})])
def test_product_refuses(code, rows, change):
    refused(lop.lop_rowwise_f8, product_op(), rows, code, **change)


def rope_op():
    return lop.lop_head_norm_rope_t(50, 4, 2, 64, 32, 0, lop.LOP_BF16, 1e-6, 1.0, A, 256, 64, A, 128, 64, A, 256, 64, A, 128, 64, A, A, A, A)


@pytest.mark.parametrize("code,rows,change", [
    (ARG, (0, 9), dict(q=None)), (ARG, (0, 9), dict(k=None)), (ARG, (0, 9), dict(q_out=None)), (ARG, (0, 9), dict(k_out=None)), (ARG, (0, 9), dict(positions=None)),
    (ARG, (0, 9), dict(freq=None)), (ARG, (0, 9), dict(q=A + 8)), (ARG, (0, 9), dict(k_out=A + 2)), (ARG, (0, 9), dict(q_weight=A + 4)), (ARG, (0, 9), dict(freq=A + 4)),
    (ARG, (0, 9), dict(positions=A + 1)), (ARG, (0, 9), dict(q_head=60)), (ARG, (0, 9), dict(k_token=-128)), (ARG, (0, 9), dict(q_out_head=56)), (ARG, (0, 9), dict(k_out_token=0)), (ARG, (0, 9), dict(eps=-1.0)), (ARG, (0, 9), dict(eps=float("nan"))),
    (ARG, (0, 0), dict(heads_q=0, heads_k=0)), (ARG, (0, 0), dict(heads_k=-1)), (ARG, (0, 0), dict(tokens=-1)), (ARG, (0, 0), dict(head_dim=0)), (ARG, (0, 0), dict(rot_dim=-8)),
    (UNS, (0, 9), dict(head_dim=60)), (UNS, (0, 9), dict(head_dim=264)), (UNS, (0, 9), dict(rot_dim=12)), (UNS, (0, 9), dict(dtype=3)), (SHAPE, (0, 9), dict(rot_dim=72)),
    (BAND, (0, 51), {}), (BAND, (-1, 3), {}), (BAND, (3, 2), {})])
def test_rope_refuses(code, rows, change):
    refused(lop.lop_head_norm_rope, rope_op(), rows, code, **change)


def attention_op():
    return lop.lop_attention_t(lop.LOP_BF16, 4, 2, 64, 3, 50, 90, 40, 1, 0.125, A, 256, 64, A, 128, 64, A, 128, 64, A, 256, 64, A, A, A, None, None, 0)


@pytest.mark.parametrize("code,rows,change", [
    (ARG, (0, 9), dict(q=None)), (ARG, (0, 9), dict(k=None)), (ARG, (0, 9), dict(v=None)), (ARG, (0, 9), dict(out=None)), (ARG, (0, 9), dict(q_offsets=None)),
    (ARG, (0, 9), dict(k_begin=None)), (ARG, (0, 9), dict(k_end=None)), (ARG, (0, 9), dict(q=A + 8)), (ARG, (0, 9), dict(v=A + 2)), (ARG, (0, 9), dict(k_end=A + 2)),
    (ARG, (0, 9), dict(lse=A + 1)), (ARG, (0, 9), dict(workspace=A + 8)), (ARG, (0, 9), dict(q_token=100)), (ARG, (0, 9), dict(out_head=-64)), (ARG, (0, 9), dict(out_head=0)), (ARG, (0, 9), dict(out_token=56)), (ARG, (0, 9), dict(k_token=56)),
    (ARG, (0, 9), dict(v_token=0)), (ARG, (0, 9), dict(scale=0.0)), (ARG, (0, 9), dict(scale=-1.0)), (ARG, (0, 9), dict(scale=float("inf"))), (ARG, (0, 9), dict(scale=float("nan"))),
    (ARG, (0, 0), dict(heads_k=0)), (ARG, (0, 0), dict(seqs=-1)), (ARG, (0, 0), dict(rows_q=-1)), (ARG, (0, 0), dict(rows_k=-1)), (ARG, (0, 0), dict(max_keys=-1)),
    (ARG, (0, 0), dict(head_dim=0)), (UNS, (0, 9), dict(head_dim=60)), (UNS, (0, 9), dict(head_dim=264)), (UNS, (0, 9), dict(dtype=2)), (UNS, (0, 9), dict(k_token=1 << 24)),
    (UNS, (0, 9), dict(rows_q=(1 << 31) - 1)), (SHAPE, (0, 9), dict(heads_q=5)), (BAND, (0, 51), {}), (BAND, (-1, 9), {}), (BAND, (9, 8), {})])
def test_attention_refuses(code, rows, change):
    refused(lop.lop_attention, attention_op(), rows, code, **change)


def test_packed_descriptors_are_the_structures():
    for packed, structure in ((lop._QUANTIZE, lop.lop_quantize_t), (lop._ROWWISE_F8, lop.lop_rowwise_f8_t),
                              (lop._HEAD_NORM_ROPE, lop.lop_head_norm_rope_t), (lop._ATTENTION, lop.lop_attention_t)):
        assert packed.size == ctypes.sizeof(structure)
        values = [i + 1 for i in range(len(structure._fields_))]
        op = structure.from_buffer_copy(packed.pack(*values))
        assert [getattr(op, name) for name, _ in structure._fields_] == values


def test_empty_bands_enqueue_nothing():
    """No GPU here: a launch would be an error."""
    lop.lop_quantize_blocks(quantize_op(), (7, 7))
    lop.lop_rowwise_f8(product_op(), (100, 100))
    lop.lop_head_norm_rope(rope_op(), (0, 0))
    lop.lop_attention(attention_op(), (50, 50))
    op = attention_op()
    op.seqs = 0
    lop.lop_attention(op, (0, 50))


def test_attention_workspace():
    op = attention_op()
    assert lop.lop_attention_workspace(op, (0, 50)) == 0            # 40 keys are not cut
    op.max_keys = 1 << 20
    n = lop.lop_attention_workspace(op, (0, 50))
    assert n > 0 and n % (50 * 4 * 66 * 4) == 0 and n // (50 * 4 * 66 * 4) <= 64
    assert lop.lop_attention_workspace(op, (10, 10)) == 0
    op.q = op.k = op.v = op.out = op.q_offsets = op.k_begin = op.k_end = None    # sizes only
    assert lop.lop_attention_workspace(op, (0, 50)) == n
    op.rows_q, op.seqs = 100000, 1                                  # enough rows to fill the GPU
    assert lop.lop_attention_workspace(op, (0, 100000)) == 0
    with pytest.raises(lop.LopError) as e:
        lop.lop_attention_workspace(op, (0, 100001))
    assert e.value.code == BAND
    with pytest.raises(lop.LopError) as e:
        lop._check(lop._lib.lop_attention_workspace(None, 1 << 32, None), "")
    assert e.value.code == ARG
    for fn in (lop._lib.lop_quantize_blocks, lop._lib.lop_rowwise_f8, lop._lib.lop_head_norm_rope, lop._lib.lop_attention):
        assert fn(None, 1 << 32, None) == ARG


# ------------------------------------------------------------------ pins of the plain forms

def test_plain_e4m3_is_torchs():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal(4000) * np.exp2(rng.integers(-12, 9, 4000)), np.arange(-448, 449), [2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -11, 0.0, 1.0625, 1.1875]])
    x = x[np.abs(x) <= 448].astype(np.float32)
    np.testing.assert_array_equal(plain.round_e4m3(x), torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy())


def test_plain_quantize_holds_what_it_says():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((5, 300)).astype(np.float32)
    q, s = plain.quantize(x, 1)
    assert q.shape == x.shape and s.shape == (5, 3)
    np.testing.assert_allclose(s[2, 1] * 448, np.abs(x[2, 128:256]).max(), rtol=1e-6)
    back = q * np.repeat(s, 128, 1)[:, :300]
    assert np.all(np.abs(back - x) <= np.maximum(np.abs(x) * (2.0 ** -4 + 1e-6), np.repeat(s, 128, 1)[:, :300] * 2.0 ** -10 * 1.001))
    q, s = plain.quantize(x, 128)
    assert s.shape == (1, 3) and np.abs(q).max() == 448
    q, s = plain.quantize(np.zeros((2, 16), np.float32), 1)
    assert (q == 0).all() and (s == np.float32(2.0 ** -64 / 448)).all()


def test_plain_product_on_whole_numbers():
    x, w = np.arange(-6, 6).reshape(2, 6) % 5, np.arange(18).reshape(3, 6) % 4
    y, size = plain.product(x, np.array([[2.0], [0.5]]), w, np.array([[4.0]]), np.array([1.0, 2.0, 3.0]), "none", np.ones((2, 3)))
    np.testing.assert_array_equal(y, (x @ w.T) * np.array([[8.0], [2.0]]) + [1, 2, 3] + 1)
    assert (size >= np.abs(y)).all()


@pytest.mark.parametrize("interleaved", [False, True])
def test_plain_rope_turns(interleaved):
    rng = np.random.default_rng(2)
    x = rng.standard_normal((3, 2, 16))
    freq = np.array([0.5, 0.25, 0.125], np.float32)
    y, size = plain.norm_rope(x, np.array([0, 1, 9]), freq, None, 0.0, interleaved, 1.0)
    np.testing.assert_allclose(y[0], x[0])
    np.testing.assert_allclose(np.linalg.norm(y, axis=-1), np.linalg.norm(x, axis=-1))
    np.testing.assert_array_equal(y[..., 6:], x[..., 6:])
    a, b = (0, 1) if interleaved else (0, 3)
    z = (x[2, 1, a] + 1j * x[2, 1, b]) * np.exp(4.5j)
    np.testing.assert_allclose([y[2, 1, a], y[2, 1, b]], [z.real, z.imag])
    assert (size + 1e-12 >= np.abs(y)).all()
    n, _ = plain.norm_rope(x, None, None, np.full(16, 2.0), 0.0, interleaved, 1.0)
    np.testing.assert_allclose((n ** 2).mean(-1), 4.0)


@pytest.mark.parametrize("causal", [True, False])
def test_plain_attention_is_torchs(causal):
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((9, 4, 8)), rng.standard_normal((20, 2, 8)), rng.standard_normal((20, 2, 8))
    out, lse, size, _ = plain.attention(q, k, v, [1, 4, 8], [2, 12], [9, 15], 0.3, causal)
    for i, (a, b, c, e) in enumerate([(1, 4, 2, 9), (4, 8, 12, 15)]):
        nq, nk = b - a, e - c
        qq, kk, vv = (torch.from_numpy(t).transpose(0, 1) for t in (q[a:b], np.repeat(k[c:e], 2, 1), np.repeat(v[c:e], 2, 1)))
        s = 0.3 * qq @ kk.transpose(1, 2)
        if causal:
            s = s.masked_fill(torch.ones(nq, nk).tril(nk - nq) == 0, -np.inf)
        some = s.isfinite().any(-1)
        want = torch.where(some[..., None], s.softmax(-1) @ vv, 0.0).transpose(0, 1)
        np.testing.assert_allclose(out[a:b], want)
        np.testing.assert_allclose(lse[:, a:b], torch.logsumexp(s, -1))
    assert np.isnan(out[0]).all() and np.isnan(out[8]).all() and (out[4, :, :] == 0).all() == causal
