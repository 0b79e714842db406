"""The operators between and inside the row-wise products of a transformer: what is measured of them, with their plain
forms.

  quantize   rows (or 128 x 128 blocks) of a matrix in 8-bit floating point (e4m3), a scale for each block of 128 columns
  product    the row-wise product y = act(x W^T + bias + residual) of operands quantized like that
  rotate     queries and keys normalized for each head and rotated by their positions, in one pass
  attend     softmax attention of packed query rows on the keys of their sequences, grouped heads

`own` chooses between the plain forms (elementary torch operations in 32 bits, angles in 64) and the library's calls.
"""
import math
import random

import torch

own = False

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 128          # columns (and, of a weight, rows) that share a scale
MOST = 448.0         # the largest e4m3 value
LEAST = 2.0 ** -64   # blocks whose largest magnitude is less are scaled as if it were this


def _ceil(a, b):
    return -(-a // b)


# ------------------------------------------------------------------ the cases

def _quantize(name, m, k, dtype, block_rows):
    return {"name": name, "op": "quantize", "m": m, "k": k, "dtype": dtype, "block_rows": block_rows}


def _product(name, m, k, n, dtype, bias=False, act="none", residual=False):
    return {"name": name, "op": "product", "m": m, "k": k, "n": n, "dtype": dtype, "bias": bias, "act": act, "residual": residual}


def _rotate(name, tokens, hq, hk, d, rot, dtype, norm=True, interleaved=False, base=1e4, far=0, stretch=1.0):
    # far: 0: the tokens of a prompt, in order; else every token is the next one of a sequence of up to that many
    return {"name": name, "op": "rotate", "tokens": tokens, "hq": hq, "hk": hk, "d": d, "rot": rot, "dtype": dtype, "norm": norm,
            "interleaved": interleaved, "base": base, "far": far, "stretch": stretch}


def _attend(name, seqs, q_lo, q_hi, k_lo, k_hi, hq, hk, d, dtype, causal=True, room=0, lse=False, lens=1):
    # lengths of a sequence: q_lo .. q_hi query rows, and k_lo .. k_hi keys in front of those (causal), or in all
    # room: keys lie in a cache with this many rows for each sequence (0: packed)
    return {"name": name, "op": "attend", "seqs": seqs, "q_lo": q_lo, "q_hi": q_hi, "k_lo": k_lo, "k_hi": k_hi, "hq": hq, "hk": hk,
            "d": d, "dtype": dtype, "causal": causal, "room": room, "lse": lse, "lens": lens}


def listed():
    return [
        # One token's activations on their way into a product: launch latency.
        _quantize("quantize token", 1, 4096, "bf16", 1),
        # The activations of a long batch of prompts.
        _quantize("quantize prompt", 16384, 4096, "bf16", 1),
        # One token through an up-projection: the weights are read once, latency counts.
        _product("product token", 1, 1024, 4096, "bf16"),
        # A serving batch, odd in every direction, with everything the epilogue does.
        _product("product ragged", 61, 2064, 4100, "f32", bias=True, act="relu", residual=True),
        # A long batch of prompts through a wide layer: the largest products.
        _product("product prompt", 16384, 4096, 16384, "bf16"),
        # The next token of a batch of long sequences.
        _rotate("rotate token", 16, 32, 8, 128, 128, "bf16", base=5e5, far=131072, stretch=8.0),
        # A long prompt, halves of the head paired.
        _rotate("rotate prompt", 16384, 32, 8, 128, 128, "bf16"),
        # Neighbours paired, part of the head, in fp32, an odd number of tokens.
        _rotate("rotate part", 3001, 20, 4, 96, 64, "f32", interleaved=True),
        # The first steps of a single conversation: as small as attention gets.
        _attend("attend token", 1, 1, 1, 40, 40, 8, 2, 64, "bf16"),
        # A serving batch that generates: one row a sequence on caches filled to different lengths.
        _attend("attend caches", 32, 1, 1, 2000, 8000, 32, 8, 128, "bf16", room=8192, lens=2),
        # Prompts of different lengths packed behind one another, in fp32, with the softmax's logarithms.
        _attend("attend packed", 6, 1, 1500, 0, 0, 12, 4, 80, "f32", lse=True, lens=3),
        # One long prompt: the largest.
        _attend("attend prompt", 1, 8192, 8192, 0, 0, 32, 8, 128, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize", "product", "product", "rotate", "attend", "attend", "attend"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "quantize":
        # Columns are a multiple of the 16 values that a vector holds; weights have blocks of rows too.
        c = _quantize("", _log(rng, 1, 16384), 16 * _log(rng, 8, 256), dtype, rng.choice([1, 1, BLOCK]))
    elif op == "product":
        c = _product("", _log(rng, 1, 16384), 16 * _log(rng, 16, 256), _log(rng, 128, 16384), dtype, rng.random() < 0.4,
                     rng.choice(["none", "none", "relu", "relu6"]), rng.random() < 0.4)
    elif op == "rotate":
        d = rng.choice([64, 80, 96, 128, 128, 256])
        hk = rng.choice([1, 2, 4, 8])
        tokens = _log(rng, 1, 16384)
        c = _rotate("", tokens, hk * rng.choice([1, 2, 4, 5]), hk, d, rng.choice([d, d, d // 2]), dtype, rng.random() < 0.7,
                    rng.random() < 0.5, rng.choice([1e4, 5e5]), rng.choice([0, 0, 4096, 131072, 1 << 20]), rng.choice([1.0, 1.0, 4.0, 32.0]))
    else:
        d = rng.choice([64, 80, 96, 128, 128, 256])
        hk = rng.choice([1, 2, 4, 8])
        hq = hk * rng.choice([1, 2, 4, 5, 7])
        hq = hq if hq <= 32 else hk * 4
        kind = rng.choice(["prompt", "prompt", "chunk", "step", "step", "all"])
        lse, lens = rng.random() < 0.3, rng.randint(1, 10 ** 6)
        if kind == "prompt":          # whole prompts, packed
            seqs = rng.choice([1, 1, 2, 4, 8])
            most = _log(rng, 1, (8192 if dtype == "bf16" else 3000) // seqs)
            c = _attend("", seqs, max(1, most // 4), most, 0, 0, hq, hk, d, dtype, True, 0, lse, lens)
        elif kind == "chunk":         # the next piece of prompts whose beginnings are in a cache
            room = _log(rng, 512, 8192)
            rows = _log(rng, 2, 256)
            c = _attend("", rng.choice([1, 2, 4]), 1, rows, 1, room - rows, hq, hk, d, dtype, True, room, lse, lens)
        elif kind == "step":          # single tokens, sometimes a few that were guessed ahead
            room = _log(rng, 64, 16384)
            rows = rng.choice([1, 1, 1, 4])
            c = _attend("", _log(rng, 1, 32), rows, rows, max(1, room // 8), room - rows, hq, hk, d, dtype, True, room, lse, lens)
        else:                         # every row sees every key of its sequence
            seqs = rng.choice([1, 3, 8])
            most = _log(rng, 2, 2048)
            c = _attend("", seqs, 1, most, 1, most, hq, hk, d, dtype, False, 0, lse, lens)
    del c["name"]
    return c


def _lengths(case):
    """Query rows and keys of each sequence."""
    r = random.Random(case["lens"])
    out = []
    for _ in range(case["seqs"]):
        nq, nk = r.randint(case["q_lo"], case["q_hi"]), r.randint(case["k_lo"], case["k_hi"])
        out.append((nq, nk + nq if case["causal"] else nk))
    return out


# ------------------------------------------------------------------ inputs

def _e4m3(x, block_rows):
    """A matrix in e4m3 and its scales, as a checkpoint or the layer before holds them."""
    m, k = x.shape
    rb, kb = _ceil(m, block_rows), _ceil(k, BLOCK)
    whole = torch.zeros(rb * block_rows, kb * BLOCK, device=x.device)
    whole[:m, :k] = x
    tiles = whole.view(rb, block_rows, kb, BLOCK)
    scale = tiles.abs().amax((1, 3)).clamp_(min=LEAST) / MOST
    q = (tiles / scale[:, None, :, None]).view(rb * block_rows, kb * BLOCK)[:m, :k].contiguous()
    return q.to(torch.float8_e4m3fn), scale


def _activations(m, k, gen):
    """Normal values with a few wide columns, as layers have them."""
    x = torch.randn(m, k, device="cuda", generator=gen)
    return x * torch.exp(0.5 * torch.randn(k, device="cuda", generator=gen))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = _TORCH[case["dtype"]]
    s = {"case": case}

    def randn(*shape):
        return torch.randn(shape, device="cuda", generator=gen)

    if case["op"] == "quantize":
        m, k = case["m"], case["k"]
        s["x"] = _activations(m, k, gen).to(dt)
        s["q"] = torch.empty(m, k, dtype=torch.float8_e4m3fn, device="cuda")
        # (scales of a column of blocks next to one another, as the product reads them)
        s["scale"] = torch.empty(_ceil(k, BLOCK), _ceil(m, case["block_rows"]), device="cuda").t()
    elif case["op"] == "product":
        m, k, n = case["m"], case["k"], case["n"]
        s["x"], scale = _e4m3(_activations(m, k, gen), 1)
        s["x_scale"] = scale.t().contiguous().t()
        s["w"], s["w_scale"] = _e4m3(randn(n, k) / math.sqrt(k), BLOCK)
        s["bias"] = randn(n) * 0.1 if case["bias"] else None
        s["residual"] = randn(m, n).to(dt) if case["residual"] else None
        s["y"] = torch.empty(m, n, dtype=dt, device="cuda")
    elif case["op"] == "rotate":
        t, hq, hk, d, rot = (case[x] for x in ("tokens", "hq", "hk", "d", "rot"))
        # queries, keys and values of a token lie behind one another, as their common product leaves them
        qkv = randn(t, hq + 2 * hk, d).to(dt)
        s["q"], s["k"] = qkv[:, :hq], qkv[:, hq:hq + hk]
        s["q_out"], s["k_out"] = torch.empty(t, hq, d, dtype=dt, device="cuda"), torch.empty(t, hk, d, dtype=dt, device="cuda")
        s["q_weight"] = 1 + 0.1 * randn(d) if case["norm"] else None
        s["k_weight"] = 1 + 0.1 * randn(d) if case["norm"] else None
        if case["far"]:
            s["positions"] = torch.randint(0, case["far"], (t,), dtype=torch.int32, device="cuda", generator=gen)
        else:
            s["positions"] = torch.arange(t, dtype=torch.int32, device="cuda")
        # frequencies; of a longer context the slower half is slowed down further and the amplitude raised a little
        i = torch.arange(rot // 2, dtype=torch.float64)
        f = case["base"] ** (-2.0 * i / rot)
        s["freq"] = torch.where(i < rot // 4, f, f / case["stretch"]).float().cuda()
        s["amplitude"] = 1.0 + 0.1 * math.log(case["stretch"])
    else:
        hq, hk, d, room = case["hq"], case["hk"], case["d"], case["room"]
        lens = _lengths(case)
        rows = sum(a for a, _ in lens)
        begin, at = [], 0
        for i, (_, b) in enumerate(lens):
            begin.append(i * room if room else at)
            at += b
        total = room * len(lens) if room else at
        s["q"], s["k"], s["v"] = randn(rows, hq, d).to(dt), randn(total, hk, d).to(dt), randn(total, hk, d).to(dt)
        offsets = [0]
        for a, _ in lens:
            offsets.append(offsets[-1] + a)
        s["q_offsets"] = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        s["k_begin"] = torch.tensor(begin, dtype=torch.int32, device="cuda")
        s["k_end"] = torch.tensor([a + b for a, (_, b) in zip(begin, lens)], dtype=torch.int32, device="cuda")
        s["max_q"], s["max_k"] = max(a for a, _ in lens), max(b for _, b in lens)
        s["out"] = torch.empty(rows, hq, d, dtype=dt, device="cuda")
        s["lse"] = torch.empty(hq, rows, device="cuda") if case["lse"] else None
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    case = s["case"]
    return {"quantize": _run_quantize, "product": _run_product, "rotate": _run_rotate, "attend": _run_attend}[case["op"]](s, case)


def _run_quantize(s, case):
    if own:
        from paper_2507_05829_amd import lop
        lop.quantize_blocks(s["x"], case["block_rows"], q=s["q"], scale=s["scale"])
        return {"q": s["q"], "scale": s["scale"]}
    x, r = s["x"].float(), case["block_rows"]
    m, k = x.shape
    rb, kb = _ceil(m, r), _ceil(k, BLOCK)
    if m != rb * r or k != kb * BLOCK:
        x = torch.nn.functional.pad(x, (0, kb * BLOCK - k, 0, rb * r - m))
    tiles = x.view(rb, r, kb, BLOCK)
    most = tiles.abs().amax((1, 3)).clamp_(min=LEAST)
    q = (tiles * (MOST / most)[:, None, :, None]).view(rb * r, kb * BLOCK)[:m, :k]
    return {"q": q.to(torch.float8_e4m3fn), "scale": most / MOST}


def _run_product(s, case):
    if own:
        from paper_2507_05829_amd import lop
        lop.rowwise_f8(s["x"], s["x_scale"], s["w"], s["w_scale"], bias=s["bias"], act=case["act"], residual=s["residual"], y=s["y"])
        return s["y"]
    k, n = case["k"], case["n"]
    x = s["x"].float() * s["x_scale"].repeat_interleave(BLOCK, 1)[:, :k]
    w = s["w"].float() * s["w_scale"].repeat_interleave(BLOCK, 0)[:n].repeat_interleave(BLOCK, 1)[:, :k]
    y = x @ w.t()
    if s["bias"] is not None:
        y += s["bias"]
    if s["residual"] is not None:
        y += s["residual"]
    if case["act"] != "none":
        y = y.clamp_(0.0, 6.0) if case["act"] == "relu6" else y.clamp_(min=0.0)
    return y.to(s["y"].dtype)


def _plain_rotate(x, weight, cos, sin, rot, interleaved):
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6) * weight
    a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if interleaved else (y[..., :rot // 2], y[..., rot // 2:rot])
    u, v = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack((u, v), -1).flatten(-2) if interleaved else torch.cat((u, v), -1)
    return torch.cat((turned, y[..., rot:]), -1).to(x.dtype) if rot < x.shape[-1] else turned.to(x.dtype)


def _run_rotate(s, case):
    if own:
        from paper_2507_05829_amd import lop
        lop.head_norm_rope(s["q"], s["k"], s["positions"], s["freq"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=1e-6,
                           interleaved=case["interleaved"], amplitude=s["amplitude"], q_out=s["q_out"], k_out=s["k_out"])
        return {"q": s["q_out"], "k": s["k_out"]}
    angle = s["positions"].double()[:, None] * s["freq"].double()
    cos = (angle.cos() * s["amplitude"]).float()[:, None]
    sin = (angle.sin() * s["amplitude"]).float()[:, None]
    return {"q": _plain_rotate(s["q"], s["q_weight"], cos, sin, case["rot"], case["interleaved"]),
            "k": _plain_rotate(s["k"], s["k_weight"], cos, sin, case["rot"], case["interleaved"])}


def _run_attend(s, case):
    scale = case["d"] ** -0.5
    if own:
        from paper_2507_05829_amd import lop
        lop.attention(s["q"], s["k"], s["v"], s["q_offsets"], s["k_begin"], s["k_end"], scale, causal=case["causal"],
                      max_keys=s["max_k"], out=s["out"], lse=s["lse"])
        return {"out": s["out"]} if s["lse"] is None else {"out": s["out"], "lse": s["lse"]}
    # The sequences side by side, each filled up to the longest; a single one is already as it has to be.
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    dev, b, g = q.device, case["seqs"], case["hq"] // case["hk"]
    lq, lk = s["max_q"], s["max_k"]
    nq, nk = s["q_offsets"][1:] - s["q_offsets"][:-1], s["k_end"] - s["k_begin"]
    i, j = torch.arange(lq, device=dev), torch.arange(lk, device=dev)
    if b > 1 or q.shape[0] != lq or k.shape[0] != lk:
        q = q[(s["q_offsets"][:-1, None] + i).clamp_(max=q.shape[0] - 1)]
        at = (s["k_begin"][:, None] + j).clamp_(max=k.shape[0] - 1)
        k, v = k[at], v[at]
    q = q.view(b, lq, case["hk"], g, case["d"]).permute(0, 2, 3, 1, 4).reshape(b, case["hk"], g * lq, case["d"])
    k = k.view(b, lk, case["hk"], case["d"]).permute(0, 2, 3, 1)
    v = v.view(b, lk, case["hk"], case["d"]).transpose(1, 2)
    p = torch.matmul(q, k).view(b, case["hk"], g, lq, lk).mul_(scale)
    hidden = j >= nk[:, None, None]                                             # (b, 1, lk)
    if case["causal"]:
        hidden = hidden | (j > i[:, None] + (nk - nq)[:, None, None])           # (b, lq, lk)
    p.masked_fill_(hidden[:, None, None], -math.inf)
    most = p.amax(-1, keepdim=True).clamp_(min=torch.finfo(torch.float32).min)  # (rows without a key stay finite)
    total = p.sub_(most).exp_().sum(-1, keepdim=True)
    o = torch.matmul(p.view(b, case["hk"], g * lq, lk), v).view(b, case["hk"], g, lq, case["d"])
    o = o / torch.where(total > 0, total, torch.ones_like(total))
    o = o.permute(0, 3, 1, 2, 4).reshape(b, lq, case["hq"], case["d"])
    here = i < nq[:, None]
    out = {"out": (o[here] if b > 1 else o[0]).to(s["q"].dtype)}
    if case["lse"]:
        lse = (most + total.log())[..., 0].permute(0, 3, 1, 2).reshape(b, lq, case["hq"])
        out["lse"] = lse[here].t().contiguous()
    return out


# ------------------------------------------------------------------ from the definitions, in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quantize":
        x, r = s["x"].double(), case["block_rows"]
        m, k = x.shape
        q, scale = torch.empty_like(x), torch.empty(_ceil(m, r), _ceil(k, BLOCK), dtype=torch.float64, device=x.device)
        for c in range(scale.shape[1]):
            part = x[:, c * BLOCK:(c + 1) * BLOCK]
            most = torch.stack([p.abs().max() for p in part.split(r)]) if r > 1 else part.abs().max(1).values
            scale[:, c] = most.clamp(min=LEAST) / MOST
            v = part / scale[:, c].repeat_interleave(r)[:m, None]
            # e4m3: three fraction bits, exponents from -6 on, ties to even
            step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
            q[:, c * BLOCK:(c + 1) * BLOCK] = torch.round(v / step) * step
        return {"q": q, "scale": scale}
    if case["op"] == "product":
        k, y = case["k"], None
        for c in range(_ceil(k, BLOCK)):
            at = slice(c * BLOCK, (c + 1) * BLOCK)
            by = s["w_scale"][:, c].double()[torch.arange(case["n"], device="cuda") // BLOCK]
            w = s["w"][:, at].double() * by[:, None]
            x = s["x"][:, at].double() * s["x_scale"][:, c].double()[:, None]
            y = x @ w.t() if y is None else y.addmm_(x, w.t())
        if s["bias"] is not None:
            y = y + s["bias"].double()
        if s["residual"] is not None:
            y = y + s["residual"].double()
        return y if case["act"] == "none" else y.clamp(0.0, 6.0 if case["act"] == "relu6" else math.inf)
    if case["op"] == "rotate":
        rot = case["rot"]
        turn = torch.polar(torch.full((1,), s["amplitude"], dtype=torch.float64, device="cuda"),
                           s["positions"].double()[:, None, None] * s["freq"].double())
        out = {}
        for name in ("q", "k"):
            y, weight = s[name].double(), s[name + "_weight"]
            if weight is not None:
                y = y / (y.pow(2).sum(-1, keepdim=True) / y.shape[-1] + 1e-6).sqrt() * weight.double()
            pairs = y[..., :rot].unflatten(-1, (rot // 2, 2)) if case["interleaved"] else y[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
            z = z.flatten(-2) if case["interleaved"] else z.transpose(-1, -2).flatten(-2)
            out[name] = torch.cat((z, y[..., rot:]), -1)
        return out
    lens, g = _lengths(case), case["hq"] // case["hk"]
    o = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full((case["hq"], o.shape[0]), -math.inf, dtype=torch.float64, device="cuda")
    begin, at = s["k_begin"].tolist(), 0
    for i, (nq, nk) in enumerate(lens):
        seen = torch.ones(nq, nk, dtype=torch.bool, device="cuda")
        seen = seen.tril(nk - nq) if case["causal"] else seen
        some = seen.any(1)
        for h in range(case["hq"]):
            k, v = (s[x][begin[i]:begin[i] + nk, h // g].double() for x in ("k", "v"))
            z = (s["q"][at:at + nq, h].double() @ k.t()) * case["d"] ** -0.5
            z[~seen] = -math.inf
            lse[h, at:at + nq] = torch.logsumexp(z, 1)
            o[at:at + nq, h] = torch.where(some[:, None], torch.softmax(z, 1) @ v, 0.0)
        at += nq
    return {"out": o, "lse": lse} if case["lse"] else {"out": o}


def work(case):
    """Inputs once, outputs once; the operations of the products and of the visible pairs."""
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "quantize":
        m, k = case["m"], case["k"]
        return {"bytes": float(m * k * (e + 1) + 4 * _ceil(k, BLOCK) * _ceil(m, case["block_rows"])), "flops": 3.0 * m * k}
    if case["op"] == "product":
        m, k, n = case["m"], case["k"], case["n"]
        kb = _ceil(k, BLOCK)
        read = m * k + n * k + 4 * kb * (m + _ceil(n, BLOCK)) + (4 * n if case["bias"] else 0) + (e * m * n if case["residual"] else 0)
        return {"bytes": float(read + e * m * n), "flops": 2.0 * m * n * k}
    if case["op"] == "rotate":
        values = case["tokens"] * (case["hq"] + case["hk"]) * case["d"]
        return {"bytes": float(2 * e * values + 4 * case["tokens"] + 2 * case["rot"]), "flops": 10.0 * values}
    lens = _lengths(case)
    pairs = sum(sum(max(0, min(nk, nk - nq + i + 1)) for i in range(nq)) if case["causal"] else nq * nk for nq, nk in lens)
    rows, keys = sum(a for a, _ in lens), sum(b for _, b in lens)
    return {"bytes": float(e * case["d"] * (2 * rows * case["hq"] + 2 * keys * case["hk"]) + (4 * rows * case["hq"] if case["lse"] else 0)),
            "flops": 4.0 * case["d"] * case["hq"] * pairs}
