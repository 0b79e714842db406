"""The transformer operators on the GPU against their plain 64-bit forms (oracle/transformer.py)."""
import numpy as np
import pytest
import torch

from operator_cases import (TORCH, assert_near, attention_tolerance, lse_tolerance, product_tolerance, rope_tolerance, values)
from oracle import transformer as plain
from paper_2507_05829_amd import lop

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(TORCH[dtype])


def host(t):
    return t.float().cpu().numpy()


# ------------------------------------------------------------------ quantize

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("m,k", [(1, 16), (1, 4096), (3, 128), (64, 144), (65, 272), (127, 1040), (128, 256), (300, 400)])
def test_quantize(m, k, block_rows, dtype):
    rng = np.random.default_rng(m * 1000 + k)
    x = values(rng, (m, k), dtype) * np.exp2(rng.integers(-9, 9, (m, 1))).astype(np.float32)
    x[m // 2, : k // 2] = 0.0
    q, s = lop.quantize_blocks(dev(x, dtype), block_rows)
    want_q, want_s = plain.quantize(x, block_rows)
    np.testing.assert_array_equal(host(s), want_s)
    np.testing.assert_array_equal(host(q), want_q)


def test_quantize_strides_band_and_odd_values():
    rng = np.random.default_rng(1)
    x = values(rng, (50, 256), "bf16")
    x[3, 5], x[4, 130], x[5, 7], x[6] = np.nan, np.inf, -np.inf, 0.0
    x[7] *= 2.0 ** -80
    wide = torch.full((50, 256 + 64), 7.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 32:288] = dev(x, "bf16")
    q = torch.full((50, 512), 1.0, device="cuda").to(F8)
    s = torch.full((50, 5), 9.0, device="cuda")
    lop.quantize_blocks(wide[:, 32:288], 1, q=q[:, 16:272], scale=s[:, 1:3], rows=(2, 41))
    want_q, want_s = plain.quantize(x, 1)
    got_q, got_s = host(q), host(s)
    np.testing.assert_array_equal(got_q[2:41, 16:272], want_q[2:41])
    np.testing.assert_array_equal(got_s[2:41, 1:3], want_s[2:41])
    assert (got_q[:2] == 1).all() and (got_q[41:] == 1).all() and (got_q[:, :16] == 1).all() and (got_q[:, 272:] == 1).all()
    assert (got_s[:2] == 9).all() and (got_s[41:] == 9).all() and (got_s[:, 0] == 9).all() and (got_s[:, 3:] == 9).all()


# ------------------------------------------------------------------ product

def operands(rng, m, k, n):
    x, xs = plain.quantize(values(rng, (m, k), "f32"), 1)
    w, ws = plain.quantize(values(rng, (n, k), "f32", k ** -0.5), 128)
    return x.astype(np.float32), xs, w.astype(np.float32), ws


PRODUCTS = [(1, 16, 1), (1, 128, 128), (1, 1040, 257), (2, 2048, 100), (7, 144, 33), (16, 512, 1000), (17, 4096, 64), (33, 400, 130),
            (64, 1024, 512), (100, 256, 100), (129, 640, 255), (256, 384, 256), (300, 128, 700), (515, 1296, 388)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,k,n", PRODUCTS)
def test_product(m, k, n, dtype):
    rng = np.random.default_rng(m * 7 + k * 3 + n)
    x, xs, w, ws = operands(rng, m, k, n)
    bias = rng.standard_normal(n).astype(np.float32) if n % 2 else None
    res = values(rng, (m, n), dtype) if m % 3 else None
    act = ["none", "relu", "relu6"][(m + n) % 3]
    y = lop.rowwise_f8(dev(x).to(F8), dev(xs), dev(w).to(F8), dev(ws), None if bias is None else dev(bias), act,
                       None if res is None else dev(res, dtype), dtype=TORCH[dtype])
    want, size = plain.product(x, xs, w, ws, bias, act, res)
    assert_near(host(y), want, product_tolerance(want, size, k, dtype), f"{m} x {k} -> {n}")


@pytest.mark.parametrize("m", [5, 40, 300])
def test_product_strides_and_band(m):
    """Operands and results inside wider buffers, scales in either order, the residual in place, a band of rows."""
    rng = np.random.default_rng(m)
    k, n = 272, 150
    x, xs, w, ws = operands(rng, m, k, n)
    res = values(rng, (m, n), "bf16")
    xb = torch.zeros((m, 512), device="cuda").to(F8)
    xb[:, 32:32 + k] = dev(x).to(F8)
    wb = torch.zeros((n, 400), device="cuda").to(F8)
    wb[:, 16:16 + k] = dev(w).to(F8)
    yb = torch.full((m, n + 9), 5.0, dtype=torch.bfloat16, device="cuda")
    yb[:, 3:3 + n] = dev(res, "bf16")
    lo, hi = m // 3, m - 1
    want, size = plain.product(x, xs, w, ws, None, "none", res)
    for scales in (dev(xs), dev(xs.T).t(), dev(np.repeat(xs, 2, 1))[:, ::2]):
        y = yb.clone()[:, 3:3 + n]
        lop.rowwise_f8(xb[:, 32:32 + k], scales, wb[:, 16:16 + k], dev(ws.T).t(), residual=y, y=y, rows=(lo, hi))
        got = host(y)
        assert_near(got[lo:hi], want[lo:hi], product_tolerance(want, size, k, "bf16")[lo:hi], f"band of {m}")
        np.testing.assert_array_equal(got[:lo], res[:lo])
        np.testing.assert_array_equal(got[hi:], res[hi:])
    assert (yb[:, :3] == 5).all() and (yb[:, 3 + n:] == 5).all()


def test_product_odd_values_stay_in_their_rows():
    rng = np.random.default_rng(4)
    m, k, n = 40, 256, 96
    x, xs, w, ws = operands(rng, m, k, n)
    x[3, 200], xs[5, 1] = np.nan, np.inf
    w[7, 3] = np.nan
    y = host(lop.rowwise_f8(dev(x).to(F8), dev(xs), dev(w).to(F8), dev(ws), dtype=torch.float32))
    with np.errstate(invalid="ignore"):
        want, size = plain.product(x, xs, w, ws)
    clean = np.ones((m, n), bool)
    clean[[3, 5]] = False
    clean[:, 7] = False
    assert np.isnan(y[3]).all() and np.isnan(y[:, 7]).all()
    assert not np.isfinite(y[5]).any()
    assert_near(y[clean], want[clean], product_tolerance(want, size, k, "f32")[clean], "the other rows")


# ------------------------------------------------------------------ head norms and rotary positions

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,hq,hk,d,rot,norm", [(1, 1, 1, 8, 8, True), (1, 32, 8, 128, 128, True), (5, 3, 1, 64, 32, True), (9, 4, 2, 80, 40, True),
                                                     (7, 20, 4, 96, 64, False), (33, 5, 0, 128, 128, True), (3, 2, 2, 256, 256, True),
                                                     (11, 6, 3, 136, 72, True), (4200, 2, 1, 64, 64, True), (6, 4, 4, 72, 0, True)])
def test_head_norm_rope(tokens, hq, hk, d, rot, norm, interleaved, dtype):
    rng = np.random.default_rng(tokens + d + rot)
    q, k = values(rng, (tokens, hq, d), dtype), values(rng, (tokens, hk, d), dtype)
    pos = rng.integers(0, 1 << 20, tokens).astype(np.int32)
    pos[0] = (1 << 31) - 1
    freq = (5e5 ** (-2.0 * np.arange(rot // 2) / max(rot, 1))).astype(np.float32) if rot else None
    wq, wk = ((1 + 0.1 * rng.standard_normal(d)).astype(np.float32) for _ in range(2)) if norm else (None, None)
    opt = lambda a: None if a is None else dev(a)  # noqa: E731
    q_out, k_out = lop.head_norm_rope(dev(q, dtype), dev(k, dtype) if hk else None, opt(pos if rot else None), opt(freq), opt(wq),
                                      opt(wk) if hk else None, 1e-5, interleaved, 1.25)
    for got, x, w in ((q_out, q, wq), (k_out, k, wk)):
        if got is None:
            assert hk == 0
            continue
        want, size = plain.norm_rope(x, pos, freq, w, 1e-5, interleaved, 1.25)
        assert_near(host(got), want, rope_tolerance(want, size, d, dtype), f"{tokens} tokens")


def test_head_norm_rope_in_place_in_a_fused_buffer():
    """Queries and keys of a common product, in place; values and the tokens outside the band stay."""
    rng = np.random.default_rng(3)
    t, hq, hk, d = 70, 8, 2, 64
    qkv = values(rng, (t, hq + 2 * hk, d), "bf16")
    buf = dev(qkv, "bf16")
    pos, freq = np.arange(t, dtype=np.int32) + 1000, (1e4 ** (-np.arange(16) / 16.0)).astype(np.float32)
    w = (1 + 0.1 * rng.standard_normal(d)).astype(np.float32)
    q, k = buf[:, :hq], buf[:, hq:hq + hk]
    lop.head_norm_rope(q, k, dev(pos), dev(freq), dev(w), None, 1e-6, q_out=q, k_out=k, rows=(9, 61))
    got = host(buf)
    for at, weight in ((slice(0, hq), w), (slice(hq, hq + hk), None)):
        want, size = plain.norm_rope(qkv[:, at], pos, freq, weight, 1e-6, False, 1.0)
        assert_near(got[9:61, at], want[9:61], rope_tolerance(want, size, d, "bf16")[9:61], "in place")
    np.testing.assert_array_equal(got[:, hq + hk:], qkv[:, hq + hk:])
    np.testing.assert_array_equal(got[:9], qkv[:9])
    np.testing.assert_array_equal(got[61:], qkv[61:])


def test_head_norm_rope_rows_of_zeros_and_odd_values():
    d = 64
    q = np.ones((4, 2, d), np.float32)
    q[0], q[1, 0, 40], q[2, 1, 63] = 0.0, np.inf, np.nan
    freq = np.array([1.0, 0.5, 0.25, 0.125], np.float32)          # values 0..7 are rotated
    got, _ = lop.head_norm_rope(dev(q), None, dev(np.zeros(4, np.int32)), dev(freq))
    np.testing.assert_array_equal(host(got), q)                   # positions of zero, no norm: everything where it was
    got, _ = lop.head_norm_rope(dev(q), None, None, None, q_weight=dev(np.ones(d, np.float32)), eps=0.5)
    got = host(got)
    assert (got[0] == 0).all()                                    # the norm of zeros is finite
    assert np.isnan(got[2, 1]).all() and np.isfinite(got[2, 0]).all() and np.isfinite(got[3]).all()


# ------------------------------------------------------------------ attention

def attend(q, k, v, offsets, begin, end, dtype, causal=True, scale=None, rows=None, lse=True, max_keys=None, workspace=None):
    """(out, lse) of a call whose outputs were filled with 99 before."""
    scale = q.shape[2] ** -0.5 if scale is None else scale
    out = torch.full(q.shape, 99.0, dtype=TORCH[dtype], device="cuda")
    ls = torch.full((q.shape[1], q.shape[0]), 99.0, device="cuda") if lse else None
    i32 = lambda a: dev(np.asarray(a, np.int32))  # noqa: E731
    lop.attention(dev(q, dtype), dev(k, dtype), dev(v, dtype), i32(offsets), i32(begin), i32(end), scale, causal, max_keys, out, ls, workspace, rows)
    return host(out), host(ls) if lse else None


def check_attention(got, q, k, v, offsets, begin, end, dtype, causal=True, scale=None, rows=None):
    scale = q.shape[2] ** -0.5 if scale is None else scale
    out, lse = got
    want, want_lse, size, spread = plain.attention(q, k, v, offsets, begin, end, scale, causal)
    lo, hi = rows or (0, q.shape[0])
    inside = np.zeros(q.shape[0], bool)
    inside[max(lo, offsets[0]):min(hi, offsets[-1])] = True
    keys = max([e - b for b, e in zip(begin, end)] + [1])
    assert_near(out[inside], want[inside], attention_tolerance(want, size, spread, keys, q.shape[2], dtype)[inside], "out")
    assert (out[~inside] == 99).all(), "rows of no sequence, or outside the band, were written"
    if lse is not None:
        tol = lse_tolerance(want_lse, spread, keys, q.shape[2])
        assert_near(lse[:, inside], want_lse[:, inside], tol[:, inside], "lse")
        assert (lse[:, ~inside] == 99).all()


def packed(rng, lens, hq, hk, d, dtype, room=0, lead=0, behind=0):
    """Sequences of (queries, keys); `lead` and `behind`: rows of q in front of the first and behind the last."""
    nq, nk = sum(a for a, _ in lens), sum(b for _, b in lens)
    offsets = np.cumsum([lead] + [a for a, _ in lens])
    begin = np.arange(len(lens)) * room + 3 if room else np.cumsum([0] + [b for _, b in lens])[:-1]
    end = begin + [b for _, b in lens]
    rows_k = room * len(lens) + 3 if room else nk
    q = values(rng, (lead + nq + behind, hq, d), dtype)
    k, v = values(rng, (rows_k, hk, d), dtype), values(rng, (rows_k, hk, d), dtype)
    return q, k, v, offsets.tolist(), begin.tolist(), end.tolist()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d", [8, 64, 72, 96, 128, 136, 256])
def test_attention_head_sizes(d, causal, dtype):
    rng = np.random.default_rng(d)
    a = packed(rng, [(33, 70), (5, 5)], 4, 2, d, dtype)
    check_attention(attend(*a, dtype, causal), *a, dtype, causal)


LENGTHS = [[(1, 1)], [(1, 63)], [(1, 64)], [(1, 65)], [(127, 127)], [(128, 128)], [(129, 129)], [(31, 300)], [(200, 40)], [(64, 0)], [(0, 50)],
           [(1, 1), (0, 7), (3, 0), (17, 17), (0, 0), (40, 90), (1, 200)], [(1, 33)] * 70]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens", LENGTHS, ids=lambda v: "-".join(f"{a}q{b}k" for a, b in v[:3]))
def test_attention_lengths(lens, causal, dtype):
    rng = np.random.default_rng(len(lens) + lens[0][1])
    a = packed(rng, lens, 3, 1, 64, dtype, lead=2, behind=5)
    check_attention(attend(*a, dtype, causal), *a, dtype, causal)


@pytest.mark.parametrize("hq,hk", [(1, 1), (8, 8), (7, 1), (40, 8), (130, 1)])
def test_attention_head_layouts(hq, hk):
    rng = np.random.default_rng(hq)
    a = packed(rng, [(9, 20), (14, 14)], hq, hk, 64, "bf16")
    check_attention(attend(*a, "bf16"), *a, "bf16")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,d", [([(1, 3000)], 128), ([(1, 2000), (4, 1), (1, 0), (2, 1500)], 80), ([(3, 1030)] * 3, 256)])
def test_attention_cut_keys(lens, d, dtype):
    """Few rows and many keys: cut into parts and joined; also with less workspace than that takes, and with a wrong idea of the lengths."""
    rng = np.random.default_rng(d)
    a = packed(rng, lens, 4, 2, d, dtype, room=3100, lead=1, behind=1)
    q = a[0]
    op = lop.lop_attention_t(lop._TYPES[TORCH[dtype]], 4, 2, d, len(lens), q.shape[0], a[1].shape[0], 3000)
    need = lop.lop_attention_workspace(op, (0, q.shape[0]))
    assert need > 0
    check_attention(attend(*a, dtype, max_keys=3000), *a, dtype)
    check_attention(attend(*a, dtype, max_keys=700), *a, dtype)
    check_attention(attend(*a, dtype, max_keys=0), *a, dtype)
    short = torch.full((need - 4,), 255, dtype=torch.uint8, device="cuda")
    check_attention(attend(*a, dtype, max_keys=3000, workspace=short), *a, dtype)


@pytest.mark.parametrize("rows", [(0, 1), (5, 41), (40, 40), (63, 64), (100, 171)])
@pytest.mark.parametrize("max_keys", [1, 5000])
def test_attention_band(rows, max_keys):
    rng = np.random.default_rng(7)
    a = packed(rng, [(60, 60), (10, 200), (101, 150)], 6, 2, 64, "bf16")
    check_attention(attend(*a, "bf16", rows=rows, max_keys=max_keys), *a, "bf16", rows=rows)


def test_attention_strides():
    """Queries, keys and values of a common product; heads in front of tokens; an output inside a wider one."""
    rng = np.random.default_rng(8)
    t, hq, hk, d = 90, 6, 2, 64
    qkv = values(rng, (t, hq + 2 * hk, d), "bf16")
    buf = dev(qkv, "bf16")
    ofs, one, end = (dev(np.array(x, np.int32)) for x in ([0, t], [0], [t]))
    want, _, size, spread = plain.attention(qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:], [0, t], [0], [t], 0.2, True)
    tol = attention_tolerance(want, size, spread, t, d, "bf16")
    wide = torch.full((t, hq + 1, d + 8), 4.0, dtype=torch.bfloat16, device="cuda")
    lop.attention(buf[:, :hq], buf[:, hq:hq + hk], buf[:, hq + hk:], ofs, one, end, 0.2, out=wide[:, :hq, :d])
    assert_near(host(wide[:, :hq, :d]), want, tol, "out of a common buffer")
    assert (wide[:, hq] == 4).all() and (wide[:, :, d:] == 4).all()
    by_head = lambda x: x.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    out = lop.attention(by_head(buf[:, :hq]), by_head(buf[:, hq:hq + hk]), by_head(buf[:, hq + hk:]), ofs, one, end, 0.2)
    assert_near(host(out), want, tol, "heads in front of tokens")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("cut", [False, True])
def test_attention_hidden_values_do_not_matter(bad, dtype, cut):
    """Keys and values that a row does not see, later tokens and the room behind a sequence, hold what they like; those
    it sees count."""
    rng = np.random.default_rng(9)
    a = packed(rng, [(40, 40), (3, 70)], 4, 2, 64, dtype, room=100)
    q, k, v, offsets, begin, end = a
    for t in (k, v):
        for e in end:
            t[e:e + 20] = bad
        t[:begin[0]] = bad
    v[begin[0] + 30, 1, 5] = bad          # token 30 of the first sequence: rows from 30 on see it
    v[begin[1] + 68, 0] = bad
    k[begin[0] + 35, 0] = bad
    check_attention(attend(*a, dtype, max_keys=4000 if cut else 1), *a, dtype)


def test_attention_large_scores():
    """Scores far apart, and all of them far from zero."""
    rng = np.random.default_rng(10)
    q, k, v, o, b, e = packed(rng, [(30, 130)], 2, 1, 64, "f32")
    k[100] = q[3, 0] * 3
    k += 4.0
    check_attention(attend(q, k, v, o, b, e, "f32", scale=2.0), q, k, v, o, b, e, "f32", scale=2.0)


def test_attention_offsets_outside_are_cut_off():
    rng = np.random.default_rng(11)
    q, k, v, o, b, e = packed(rng, [(10, 20), (12, 30)], 2, 1, 64, "bf16")
    got = attend(q, k, v, [0, 10, 4000], [-5, 20], [20, 9999], "bf16")
    check_attention(got, q, k, v, [0, 10, 22], [0, 20], [20, 50], "bf16")
    out, lse = attend(q, k, v, [0, 10, 3], [0, 40], [20, 20], "bf16")     # an order that is none: nothing outside is touched
    assert (out[10:] == 99).all()


# ------------------------------------------------------------------ far into large tensors

def test_offsets_that_pass_32_bits():
    """The last rows of tensors of more than 4 GiB, of which only those are filled."""
    rng = np.random.default_rng(13)
    m, k, n, lo = 1100000, 4096, 48, 1099960
    x, xs, w, ws = operands(rng, m - lo, k, n)
    big, scales = torch.empty(m, k, dtype=F8, device="cuda"), torch.empty(32, m, device="cuda").t()
    big[lo:], scales[lo:] = dev(x).to(F8), dev(xs)
    y = lop.rowwise_f8(big, scales, dev(w).to(F8), dev(ws), rows=(lo, m))
    want, size = plain.product(x, xs, w, ws)
    assert_near(host(y[lo:]), want, product_tolerance(want, size, k, "bf16"), "product")
    values_in = values(rng, (m - lo, k), "bf16")
    wide = torch.empty(m, k, dtype=torch.bfloat16, device="cuda")
    wide[lo:] = dev(values_in, "bf16")
    lop.quantize_blocks(wide, q=big, scale=scales, rows=(lo, m))
    want_q, want_s = plain.quantize(values_in, 1)
    np.testing.assert_array_equal(host(big[lo:]), want_q)
    np.testing.assert_array_equal(host(scales[lo:]), want_s)
    del big
    pos, freq = torch.arange(m, dtype=torch.int32, device="cuda"), (1e4 ** (-np.arange(32) / 32.0)).astype(np.float32)
    heads = wide.view(m, 32, 128)
    lop.head_norm_rope(heads, None, pos, dev(freq), q_out=heads, rows=(lo, m))
    want, size = plain.norm_rope(values_in.reshape(-1, 32, 128), np.arange(lo, m), freq, None, 0.0, False, 1.0)
    assert_near(host(heads[lo:]), want, rope_tolerance(want, size, 128, "bf16"), "rotation")
    q, v = values(rng, (3, 32, 128), "bf16"), values(rng, (m - lo, 32, 128), "bf16")
    cache = torch.empty(m, 32, 128, dtype=torch.bfloat16, device="cuda")
    cache[lo:] = dev(v, "bf16")
    i32 = lambda a: dev(np.array(a, np.int32))  # noqa: E731
    out = lop.attention(dev(q, "bf16"), heads, cache, i32([0, 3]), i32([lo]), i32([m]), 0.1)
    want, _, size, spread = plain.attention(q, host(heads[lo:]), v, [0, 3], [0], [m - lo], 0.1, True)
    assert_near(host(out), want, attention_tolerance(want, size, spread, m - lo, 128, "bf16"), "attention")


def test_a_cache_longer_than_its_bytes_fit_32_bits():
    """One sequence of which the last key lies more than 4 GiB behind the first; nearly all weight lies on a few keys."""
    rng = np.random.default_rng(14)
    n, d = 70000, 128
    kv = torch.zeros(n, 256, d, dtype=torch.bfloat16, device="cuda")     # one key head of 256: 64 KiB from key to key
    k, v = kv[:, :1], kv[:, 1:2]
    q = values(rng, (1, 1, d), "bf16")
    v[:] = 1.0
    spikes = [3, 32767, 32768, 65535, 65536, n - 1]
    vals = values(rng, (len(spikes), d), "bf16")
    for i, s in enumerate(spikes):
        k[s, 0], v[s, 0] = dev(q[0, 0], "bf16"), dev(vals[i], "bf16")
    scale = 40.0 / float((q[0, 0] ** 2).sum())                            # the others have weights of e^-40
    i32 = lambda a: dev(np.array(a, np.int32))  # noqa: E731
    for max_keys in (0, n):
        out = lop.attention(dev(q, "bf16"), k, v, i32([0, 1]), i32([0]), i32([n]), scale, max_keys=max_keys)
        want = vals.astype(np.float64).mean(0)[None, None]
        # the others' weight, n e^-40 < 1e-12; weights and output rounded to bf16, sums of a few values of size up to 4
        assert_near(host(out), want, 2 * 2.0 ** -8 * np.abs(vals).mean(0) + 1e-5, "spikes")


# ------------------------------------------------------------------ streams, graphs, all together

def test_operators_on_another_stream_and_in_a_graph():
    """A layer's attention on a side stream, captured and replayed between other work, each replay with other inputs."""
    rng = np.random.default_rng(12)
    t, hq, hk, d, width = 50, 8, 2, 64, 256
    dt = torch.bfloat16
    w_qkv = lop.quantize_blocks(dev(values(rng, ((hq + 2 * hk) * d, width), "f32", width ** -0.5)), 128)
    w_out = lop.quantize_blocks(dev(values(rng, (width, hq * d), "f32", (hq * d) ** -0.5)), 128)
    norm = dev((1 + 0.1 * rng.standard_normal(d)).astype(np.float32))
    freq = dev((1e4 ** (-np.arange(d // 2) / (d / 2.0))).astype(np.float32))
    pos = torch.arange(t, dtype=torch.int32, device="cuda")
    ofs, begin, end = (dev(np.array(x, np.int32)) for x in ([0, 20, 50], [0, 20], [20, 50]))

    def layer(x):
        qkv = lop.rowwise_f8(*lop.quantize_blocks(x), *w_qkv).view(t, hq + 2 * hk, d)
        q, k = lop.head_norm_rope(qkv[:, :hq], qkv[:, hq:hq + hk], pos, freq, norm, norm)
        o = lop.attention(q, k, qkv[:, hq + hk:], ofs, begin, end, d ** -0.5, max_keys=4096)
        return lop.rowwise_f8(*lop.quantize_blocks(o.view(t, hq * d)), *w_out, residual=x)

    def plain_layer(x):
        """The same with every intermediate result rounded to bf16 as the layer's are."""
        b16 = lambda a: torch.from_numpy(a.astype(np.float32)).to(dt).float().numpy()  # noqa: E731
        f = [host(a) for a in (*w_qkv, *w_out)]
        qkv = b16(plain.product(*[a.astype(np.float32) for a in plain.quantize(x, 1)], f[0], f[1])[0]).reshape(t, hq + 2 * hk, d)
        p, fr, nw = pos.cpu().numpy(), host(freq), host(norm)
        q, k = (b16(plain.norm_rope(y, p, fr, nw, 1e-6, False, 1.0)[0]) for y in (qkv[:, :hq], qkv[:, hq:hq + hk]))
        o = b16(plain.attention(q, k, qkv[:, hq + hk:], [0, 20, 50], [0, 20], [20, 50], d ** -0.5, True)[0])
        return plain.product(*[a.astype(np.float32) for a in plain.quantize(o.reshape(t, -1), 1)], f[2], f[3], residual=x)[0]

    x = torch.empty(t, width, dtype=dt, device="cuda")
    inputs = [dev(values(rng, (t, width), "bf16"), "bf16") for _ in range(4)]
    eager = [layer(i) for i in inputs]
    # Roundings of 2^-8 at five places and of 2^-4 at two change what the next operator gets: in norm 2 x 2^-4 / sqrt(3) at most.
    for i, e in zip(inputs, eager):
        want = plain_layer(host(i))
        assert np.linalg.norm(host(e) - want) <= 2 * 2.0 ** -4 / 3 ** 0.5 * np.linalg.norm(want - host(i))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for i, e in zip(inputs, eager):
            assert torch.equal(layer(i), e)
        graph = torch.cuda.CUDAGraph()
        x.copy_(inputs[0])
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            y = layer(x)
    torch.cuda.synchronize()
    for i, e in list(zip(inputs, eager)) * 2:
        x.copy_(i)
        torch.cuda.synchronize()
        graph.replay()
        assert torch.equal(layer(i), e)      # the program's own work between replays
        torch.cuda.synchronize()
        assert torch.equal(y, e)


def test_operators_refuse_what_does_not_fit():
    dt = torch.bfloat16
    q, k = torch.zeros(4, 4, 64, dtype=dt, device="cuda"), torch.zeros(4, 2, 64, dtype=dt, device="cuda")
    o, b, e = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 4], [0], [4]))
    lop.attention(q, k, k, o, b, e, 1.0)
    for bad in (lambda: lop.attention(q, k.float(), k, o, b, e, 1.0), lambda: lop.attention(q.cpu(), k, k, o, b, e, 1.0),
                lambda: lop.attention(q, k, k, o.long(), b, e, 1.0), lambda: lop.attention(q, k, k, b, b, e, 1.0),
                lambda: lop.attention(q, k, k[:3], o, b, e, 1.0), lambda: lop.attention(q.clone().requires_grad_(), k, k, o, b, e, 1.0),
                lambda: lop.attention(q.transpose(1, 2), k, k, o, b, e, 1.0), lambda: lop.attention(q, k, k, o, b, e, 1.0, lse=torch.zeros(4, 5, device="cuda")),
                lambda: lop.quantize_blocks(q[0].half()), lambda: lop.quantize_blocks(q[0], 64), lambda: lop.quantize_blocks(q[0], q=torch.zeros(4, 64, device="cuda")),
                lambda: lop.head_norm_rope(q, k, o, None), lambda: lop.head_norm_rope(q, k[:3], None, None)):
        with pytest.raises(ValueError):
            bad()
    for bad, code in ((lambda: lop.attention(q, k, k, o, b, e, 0.0), lop.LOP_ERR_INVALID_ARG), (lambda: lop.attention(q[:, :3], k, k, o, b, e, 1.0), lop.LOP_ERR_SHAPE),
                      (lambda: lop.attention(q[..., 4:], k[..., 4:], k[..., 4:], o, b, e, 1.0), lop.LOP_ERR_UNSUPPORTED),
                      (lambda: lop.attention(q[..., 4:12], k[..., 4:12], k[..., 4:12], o, b, e, 1.0), lop.LOP_ERR_INVALID_ARG),
                      (lambda: lop.attention(q, k, k, o, b, e, 1.0, rows=(0, 5)), lop.LOP_ERR_BAND_RANGE),
                      (lambda: lop.quantize_blocks(q[0][:, :40]), lop.LOP_ERR_UNSUPPORTED)):
        with pytest.raises(lop.LopError) as err:
            bad()
        assert err.value.code == code


# ------------------------------------------------------------------ calls that share something

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,hq,hk,d", [(700, 20, 6, 128), (1300, 20, 6, 128), (4200, 20, 6, 128), (2000, 9, 0, 256), (3000, 40, 3, 64)])
def test_head_norm_rope_several_heads_in_turn(tokens, hq, hk, d, dtype):
    """Wavefronts that go through some of a token's heads, or all, the last of them fewer."""
    rng = np.random.default_rng(tokens + hq)
    qk = values(rng, (tokens, hq + hk, d), dtype)
    pos = rng.integers(0, 1 << 17, tokens).astype(np.int32)
    freq = (1e6 ** (-2.0 * np.arange(d // 2) / d)).astype(np.float32)
    w = (1 + 0.1 * rng.standard_normal(d)).astype(np.float32)
    x = dev(qk, dtype)
    q_out, k_out = lop.head_norm_rope(x[:, :hq], x[:, hq:] if hk else None, dev(pos), dev(freq), dev(w), dev(w) if hk else None, 1e-6)
    want, size = plain.norm_rope(qk, pos, freq, w, 1e-6, False, 1.0)
    got = host(q_out if k_out is None else torch.cat((q_out, k_out), 1))
    assert_near(got, want, rope_tolerance(want, size, d, dtype), f"{tokens} tokens")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("max_keys", [None, 10])
def test_attention_sequences_that_share_keys(dtype, max_keys):
    """The same keys for several sequences, whole, in part or overlapping, and one without any."""
    rng = np.random.default_rng(21)
    q, k, v, *_ = packed(rng, [(9, 900)], 6, 2, 72, dtype)
    offsets, begin, end = [0, 1, 4, 5, 8, 9], [0, 0, 130, 0, 700], [900, 900, 830, 0, 900]
    check_attention(attend(q, k, v, offsets, begin, end, dtype, max_keys=max_keys), q, k, v, offsets, begin, end, dtype)


def test_calls_at_once_on_two_streams():
    """Each with its own workspace and outputs: what one call at a time gives, bit for bit."""
    rng = np.random.default_rng(22)
    jobs = []
    for dtype, d in (("bf16", 128), ("f32", 64)):
        q, k, v, offsets, begin, end = packed(rng, [(1, 3000), (2, 1700)], 8, 2, d, dtype)
        args = [dev(a, dtype) for a in (q, k, v)] + [dev(np.array(a, np.int32)) for a in (offsets, begin, end)]
        jobs.append(lambda args=args, d=d: lop.attention(*args, d ** -0.5))
    for m in (1, 40, 600):
        x, w = lop.quantize_blocks(dev(values(rng, (m, 1040), "f32"))), lop.quantize_blocks(dev(values(rng, (400, 1040), "f32")), 128)
        jobs.append(lambda x=x, w=w: lop.rowwise_f8(*x, *w))
    alone = [job() for job in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for i in range(12):
        for j, job in enumerate(jobs):
            with torch.cuda.stream(streams[(i + j) % 2]):
                got.append((j, job()))
    torch.cuda.synchronize()
    for j, y in got:
        assert torch.equal(y, alone[j])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_cache_that_grows_between_replays(dtype):
    """One captured step whose keys are cut into parts; its offsets, inputs and cache change between the replays, the graph does not."""
    rng = np.random.default_rng(23)
    room, hq, hk, d = 2100, 8, 2, 64
    k, v = (values(rng, (2 * room, hk, d), dtype) for _ in range(2))
    k_dev, v_dev = dev(k, dtype), dev(v, dtype)
    q_dev = torch.zeros(2, hq, d, dtype=TORCH[dtype], device="cuda")
    ofs, begin = dev(np.array([0, 1, 2], np.int32)), dev(np.array([0, room], np.int32))
    end = dev(np.array([1, room], np.int32))
    out = torch.empty_like(q_dev)
    lse = torch.empty(hq, 2, device="cuda")

    def step():
        lop.attention(q_dev, k_dev, v_dev, ofs, begin, end, d ** -0.5, max_keys=room, out=out, lse=lse)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()
    for lens in ((1, 0), (0, 2100), (700, 31), (2100, 2100), (64, 65)):
        q = values(rng, (2, hq, d), dtype)
        q_dev.copy_(dev(q, dtype))
        end.copy_(dev(np.array([lens[0], room + lens[1]], np.int32)))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got, got_lse = out.clone(), lse.clone()
        ends = [lens[0], room + lens[1]]
        check_attention((host(got), host(got_lse)), q, k, v, [0, 1, 2], [0, room], ends, dtype)
        step()
        torch.cuda.synchronize()
        assert torch.equal(out, got) and torch.equal(lse, got_lse)
