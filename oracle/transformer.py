"""Plain 64-bit forms of the operators beside the row-wise products of a transformer, written from their definitions: block
quantization to e4m3, the product of quantized operands, head norms with rotary positions, and softmax attention of packed
sequences. numpy only; nothing here is fast."""
import numpy as np

BLOCK = 128


def _blocks(a, rows):
    """Each entry of a scale matrix repeated over its block, cut to the rows and columns that `rows` = (m, k, block_rows) has."""
    m, k, block_rows = rows
    return np.repeat(np.repeat(a, block_rows, 0)[:m], BLOCK, 1)[:, :k]


def round_e4m3(x):
    """Nearest e4m3 value (three fraction bits, exponents from -6 on, at most 448), ties to even; float64 in and out."""
    x = np.asarray(x, np.float64)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6)))
        step = np.exp2(e - 3)
        return np.rint(x / step) * step


def quantize(x, block_rows):
    """(values, scales) of a float32 matrix: the two roundings of the definition (448 / a, and the product with it) are float32."""
    x = np.asarray(x, np.float32)
    m, k = x.shape
    rb, kb = -(-m // block_rows), -(-k // BLOCK)
    a = np.zeros((rb, kb), np.float32)
    for i in range(rb):
        for j in range(kb):
            part = np.abs(x[i * block_rows:(i + 1) * block_rows, j * BLOCK:(j + 1) * BLOCK])
            part = part[~np.isnan(part)]
            a[i, j] = max(part.max() if part.size else 0.0, 2.0 ** -64)
    with np.errstate(invalid="ignore", over="ignore"):
        by = _blocks(np.float32(448.0) / a, (m, k, block_rows))
        return round_e4m3(x * by), a / np.float32(448.0)


def product(x, x_scale, w, w_scale, bias=None, act="none", residual=None):
    """(y, sum of the magnitudes of its products): the second scales what sums in fewer bits may be off by."""
    m, k = x.shape
    n = w.shape[0]
    a = x.astype(np.float64) * _blocks(x_scale.astype(np.float64), (m, k, 1))
    b = w.astype(np.float64) * _blocks(w_scale.astype(np.float64), (n, k, BLOCK))
    y = a @ b.T
    size = np.abs(a) @ np.abs(b).T
    if bias is not None:
        y, size = y + bias.astype(np.float64), size + np.abs(bias.astype(np.float64))
    if residual is not None:
        y, size = y + residual.astype(np.float64), size + np.abs(residual.astype(np.float64))
    return (y if act == "none" else np.clip(y, 0.0, 6.0 if act == "relu6" else np.inf)), size


def norm_rope(x, positions, freq, weight, eps, interleaved, amplitude):
    """(y, size): x (tokens, heads, d); size bounds the two terms that each value of y is the sum of."""
    y = x.astype(np.float64)
    if weight is not None:
        y = y / np.sqrt((y ** 2).mean(-1, keepdims=True) + eps) * weight.astype(np.float64)
    size = np.abs(y)
    if freq is None:
        return y, size
    half = len(freq)
    angle = positions.astype(np.float64)[:, None, None] * freq.astype(np.float64)
    c, s = np.cos(angle) * amplitude, np.sin(angle) * amplitude
    ia = np.arange(half) * 2 if interleaved else np.arange(half)
    ib = ia + 1 if interleaved else ia + half
    out, bound = y.copy(), size.copy()
    a, b = y[..., ia], y[..., ib]
    out[..., ia], out[..., ib] = a * c - b * s, a * s + b * c
    bound[..., ia] = bound[..., ib] = (np.abs(a) + np.abs(b)) * abs(amplitude)
    return out, bound


def attention(q, k, v, q_offsets, k_begin, k_end, scale, causal):
    """(out, lse, size, spread): q (rows, heads_q, d). size: the weighted mean of |v|, spread: scale * the largest sum of |q_i k_i| of a
    row. Rows of no sequence are NaN in out and lse, rows that see no key 0 and -inf."""
    rows, hq, d = q.shape
    g = hq // k.shape[1]
    out = np.full((rows, hq, d), np.nan)
    lse = np.full((hq, rows), np.nan)
    size, spread = np.zeros((rows, hq, d)), np.zeros((rows, hq))
    q, k, v = (t.astype(np.float64) for t in (q, k, v))
    for i in range(len(k_begin)):
        q0, q1, k0, k1 = int(q_offsets[i]), int(q_offsets[i + 1]), int(k_begin[i]), int(k_end[i])
        nq, nk = q1 - q0, max(0, k1 - k0)
        for r in range(nq):
            sees = min(nk, max(0, nk - nq + r + 1)) if causal else nk
            for h in range(hq):
                at = (q0 + r, h)
                if sees == 0:
                    out[at], lse[h, q0 + r] = 0.0, -np.inf
                    continue
                kk, vv = k[k0:k0 + sees, h // g], v[k0:k0 + sees, h // g]
                with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
                    s = scale * (kk @ q[at])
                    m = s.max()
                    p = np.exp(s - (m if np.isfinite(m) else 0.0))
                    out[at] = (p @ vv) / p.sum()
                    lse[h, q0 + r] = m + np.log(p.sum())
                    size[at] = (p @ np.abs(vv)) / p.sum()
                    spread[at] = scale * (np.abs(kk) @ np.abs(q[at])).max()
    return out, lse, size, spread
