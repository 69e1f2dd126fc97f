"""The operators around an 8-bit stale K/V cache, as cases to be timed and compared.

Three kinds of calls, in the order in which a band's step makes them:

  rotary     rotary positions of a band's tokens on a (frames, rows, columns)
             grid, applied to Q and to K (K inside the band's K/V buffer)
  kv_cache   the band's K/V written into the 8-bit cache (e4m3 values, one
             power-of-two scale per head and token), and the whole cache read
             back into a K/V buffer of the operand type
  attention  the band's queries over the whole image: its own K/V fresh, every
             other token's from the 8-bit cache

`own` false: the operators in elementary torch operations, 32 bits throughout
(64 for angles).  `own` true: the package's entry points.  Sizes are those of
seeded_inputs/configs.py (the tiny fp32 model, DiT-S/2 at 256px, DiT-XL/2 at
512, 1024 and 2048px) and generic ones between them.
"""
import math

import torch

own = False

DEV = "cuda:0"


# ---- the cases ---------------------------------------------------------------

def _rotary(name, B, heads, d, grid, token_begin, n_tok, channels, theta, origin, step, interleaved, dtype):
    return {"name": name, "kind": "rotary", "B": B, "heads": heads, "head_dim": d, "frames": grid[0],
            "rows": grid[1], "cols": grid[2], "token_begin": token_begin, "n_tok": n_tok, "ch_t": channels[0],
            "ch_h": channels[1], "ch_w": channels[2], "theta": theta, "origin": origin, "step": step,
            "interleaved": interleaved, "dtype": dtype}


def _kv_cache(name, B, heads, d, tokens, tok_offset, n_tok, dtype):
    return {"name": name, "kind": "kv_cache", "B": B, "heads": heads, "head_dim": d, "tokens": tokens,
            "tok_offset": tok_offset, "n_tok": n_tok, "dtype": dtype}


def _attention(name, B, heads, d, n_q, n_kv, fresh_begin, n_fresh, dtype):
    return {"name": name, "kind": "attention", "B": B, "heads": heads, "head_dim": d, "n_q": n_q,
            "n_kv": n_kv, "fresh_begin": fresh_begin, "n_fresh": n_fresh, "dtype": dtype}


def listed():
    return [
        # the tiny fp32 model's half image: a call that is all launch and latency
        _rotary("rotary_tiny_f32", 1, 4, 32, (1, 8, 8), 0, 32, (0, 16, 16), 1e4, 0.0, 1.0, True, "f32"),
        # DiT-XL/2 at 1024px with guidance, the 40% band in the image's middle: 36 channels for each of two axes,
        # positions counted from the image's centre
        _rotary("rotary_xl1024_band40", 2, 16, 72, (1, 64, 64), 19 * 64, 26 * 64, (0, 36, 36), 1e4, -31.5, 1.0,
                True, "bf16"),
        # a video latent, 13 frames of 45 x 80 tokens, 128-channel heads, three axes, halves of an axis paired
        _rotary("rotary_video_d128", 1, 16, 128, (13, 45, 80), 0, 13 * 45 * 80, (16, 56, 56), 256.0, 0.0, 0.5,
                False, "bf16"),
        # the tiny fp32 model's exchange
        _kv_cache("cache_tiny_f32", 1, 4, 32, 64, 0, 32, "f32"),
        # DiT-XL/2 at 1024px: the 40% band into the cache, the image's K/V out of it
        _kv_cache("cache_xl1024_band40", 2, 16, 72, 4096, 19 * 64, 26 * 64, "bf16"),
        # every row at 2048px (a synchronous warm-up step's exchange)
        _kv_cache("cache_xl2048_all", 2, 16, 72, 16384, 0, 16384, "bf16"),
        # DiT-S/2 at 256px, its 40% band: a small model, latency
        _attention("attn_s2_256_band40", 1, 6, 64, 96, 256, 80, 96, "bf16"),
        # one row of a 45 x 45 grid, 128-channel heads: odd counts, a band that starts and ends inside every tile
        _attention("attn_d128_odd", 2, 8, 128, 45, 2025, 1035, 45, "bf16"),
        # fp32 heads (reference runs), every key from the cache
        _attention("attn_f32_cached", 1, 4, 32, 512, 1024, 0, 0, "f32"),
        # DiT-XL/2 at 512px, 12 of 32 rows
        _attention("attn_xl512_band12", 2, 16, 72, 384, 1024, 320, 384, "bf16"),
        # DiT-XL/2 at 1024px, the 40% band: one device's share of a production sampler
        _attention("attn_xl1024_band40", 2, 16, 72, 26 * 64, 4096, 19 * 64, 26 * 64, "bf16"),
        # 48 of 128 rows at 2048px: the longest key stream
        _attention("attn_xl2048_band48", 2, 16, 72, 48 * 128, 16384, 40 * 128, 48 * 128, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _grid(rng, lo, hi, most):
    rows = _log_int(rng, lo, hi)
    cols = rows if rng.random() < 0.5 else _log_int(rng, lo, hi)
    while rows * cols > most:
        rows, cols = max(1, rows - 1), max(1, cols - 1)
    return rows, cols


def draw(rng):
    """One more case of the listed kinds' ranges."""
    kind = rng.choice(("rotary", "kv_cache", "attention", "attention"))
    f32 = rng.random() < 0.25
    dtype = "f32" if f32 else "bf16"
    d = rng.choice((32, 64, 64, 72, 72, 80, 96, 128))
    heads, B = rng.randint(1, 16), rng.randint(1, 2)
    if kind == "rotary":
        frames = rng.choice((1, 1, 1, rng.randint(2, 13)))
        rows, cols = _grid(rng, 2, 100, max(4, 40000000 // (frames * B * heads * d * (2 if f32 else 1))))
        t = 0 if frames == 1 else 2 * rng.randint(1, d // 8)
        h = 2 * rng.randint(1, (d - t) // 4)
        n = frames * rows * cols
        n_tok = _log_int(rng, 1, n)
        c = _rotary("", B, heads, d, (frames, rows, cols), rng.randint(0, n - n_tok), n_tok,
                    (t, h, 2 * rng.randint(0, (d - t - h) // 2)), rng.choice((100.0, 256.0, 1e4, 1e6)),
                    rng.choice((0.0, 0.0, -0.5 * rows, 4096.0)), rng.choice((1.0, 1.0, 0.5, 0.25)),
                    rng.random() < 0.5, dtype)
    elif kind == "kv_cache":
        rows, cols = _grid(rng, 2, 128, 16384 // (2 if f32 else 1))
        n_tok = cols * _log_int(rng, 1, rows) if rng.random() < 0.7 else _log_int(rng, 1, rows * cols)
        c = _kv_cache("", B, heads, d if d <= 80 else 72, rows * cols, rng.randint(0, rows * cols - n_tok), n_tok,
                      dtype)
    else:
        rows, cols = _grid(rng, 4, 32 if f32 else 96, 1024 if f32 else 9216)
        n = rows * cols
        n_q = cols * _log_int(rng, 1, rows) if rng.random() < 0.8 else _log_int(rng, 1, 64)
        n_q = min(n_q, n, 512 if f32 else max(1, 10 ** 11 // (B * heads * n * d)))
        fresh = rng.random() < 0.7
        c = _attention("", B, heads, d, n_q, n, rng.randint(0, n - n_q) if fresh else 0, n_q if fresh else 0, dtype)
    del c["name"]
    return c


# ---- inputs --------------------------------------------------------------------

def _td(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 29)
    return g


def _kv_buffer(g, c, n):
    """K and V of n tokens as the projection leaves them: some channels and some tokens larger than others, one
    fp32 value for each (branch, head, token, channel), then the buffer layout K [heads][n][d], V^T [heads][d][n]."""
    B, heads, d = c["B"], c["heads"], c["head_dim"]
    k = torch.randn((B, heads, n, d), generator=g, device=DEV)
    k *= torch.exp(0.5 * torch.randn((1, heads, 1, d), generator=g, device=DEV))
    v = torch.randn((B, heads, n, d), generator=g, device=DEV)
    v *= torch.exp(torch.randn((B, heads, n, 1), generator=g, device=DEV))
    return torch.cat((k.reshape(B, -1), v.transpose(2, 3).reshape(B, -1)), 1).to(_td(c)).contiguous()


def _kv_views(c, buf, n):
    """K [B, heads, n, d] and V [B, heads, n, d] of a buffer of n tokens."""
    B, heads, d = c["B"], c["heads"], c["head_dim"]
    k, vt = buf.view(B, 2, heads * n * d).unbind(1)
    return k.view(B, heads, n, d), vt.view(B, heads, d, n).transpose(2, 3)


def _exponent(x):
    """E8M0 byte per row of x: the smallest power of two s = 2^(e - 127) with max |x| <= 448 s, e at least 1."""
    bits = x.abs().amax(-1).view(torch.int32)
    return ((bits >> 23) - 8 + ((bits & 0x7FFFFF) > 0x600000).int()).clamp(min=1)


def _scale(e):
    return (e.int() << 23).view(torch.float32)


def _to_cache(values, exponents, k, v, offset):
    """K/V [B, heads, n, d] into tokens [offset, +n) of the cache (values e4m3 [B, 2, heads, N, d], E8M0 exponents
    uint8 [B, 2, heads, N])."""
    n = k.shape[2]
    for i, x in enumerate((k.float(), v.float())):
        e = _exponent(x)
        values[:, i, :, offset:offset + n] = (x / _scale(e)[..., None]).to(torch.float8_e4m3fn)
        exponents[:, i, :, offset:offset + n] = e.to(torch.uint8)


def _cache(c, g, n):
    B, heads, d = c["B"], c["heads"], c["head_dim"]
    values = torch.empty((B, 2, heads, n, d), dtype=torch.float8_e4m3fn, device=DEV)
    exponents = torch.empty((B, 2, heads, n), dtype=torch.uint8, device=DEV)
    _to_cache(values, exponents, *_kv_views(c, _kv_buffer(g, c, n), n), 0)
    return values, exponents


def prepare(case, seed):
    c = case
    g = _gen(seed)
    s = {"case": c}
    B, heads, d = c["B"], c["heads"], c["head_dim"]
    if c["kind"] == "rotary":
        n = c["n_tok"]
        s["q"] = torch.randn((B, heads, n, d), generator=g, device=DEV).to(_td(c))
        s["kv"] = _kv_buffer(g, c, n)
        s["k"] = _kv_views(c, s["kv"], n)[0]
        s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty((B, heads, n, d), dtype=_td(c), device=DEV)
    elif c["kind"] == "kv_cache":
        n, N = c["n_tok"], c["tokens"]
        s["values"], s["exponents"] = _cache(c, g, N)
        s["kv"] = _kv_buffer(g, c, n)
        s["back"] = torch.empty((B, 2 * N * heads * d), dtype=_td(c), device=DEV)
    else:
        n, N, nf = c["n_q"], c["n_kv"], c["n_fresh"]
        s["q"] = torch.randn((B, heads, n, d), generator=g, device=DEV).to(_td(c))
        s["values"], s["exponents"] = _cache(c, g, N)
        s["fresh"] = _kv_buffer(g, c, nf) if nf else None
        s["out"] = torch.empty((B, n, heads * d), dtype=_td(c), device=DEV)
    if own:
        from paper_2509_04719_amd import _lib
        code = _lib.DTYPE_CODE[c["dtype"]]
        if c["kind"] == "rotary":
            s["axes"] = _lib.rotary_axes((c["ch_t"], c["ch_h"], c["ch_w"]), (c["frames"], c["rows"], c["cols"]),
                                         theta=c["theta"], origin=(0.0, c["origin"], c["origin"]),
                                         step=(1.0, c["step"], c["step"]), interleaved=c["interleaved"])
        else:
            s["cache"] = _lib.quantized_kv(s["values"], s["exponents"])
            if c["kind"] == "attention":
                need = _lib.attention_quantized_workspace_bytes(B, heads, c["n_q"], c["n_kv"], d, code)
                s["workspace"] = torch.empty(need, dtype=torch.uint8, device=DEV) if need else None
    return s


# ---- one pass ------------------------------------------------------------------

def _angles(c):
    """Angle (64 bits) of every token of the band and every rotated pair, with the pairs' channels."""
    n = torch.arange(c["token_begin"], c["token_begin"] + c["n_tok"], device=DEV)
    index = (n // (c["rows"] * c["cols"]), n // c["cols"] % c["rows"], n % c["cols"])
    place = ((0.0, 1.0), (c["origin"], c["step"]), (c["origin"], c["step"]))
    phi, first, second, base = [], [], [], 0
    for idx, ch, (origin, step) in zip(index, (c["ch_t"], c["ch_h"], c["ch_w"]), place):
        i = torch.arange(ch // 2, device=DEV)
        freq = c["theta"] ** (-2.0 * i.double() / max(ch, 1))
        phi.append(((idx.double() + origin) * step)[:, None] * freq)
        first.append(base + (2 * i if c["interleaved"] else i))
        second.append(base + (2 * i + 1 if c["interleaved"] else i + ch // 2))
        base += ch
    return torch.cat(phi, 1), torch.cat(first), torch.cat(second)


def _run_plain(s):
    c = s["case"]
    if c["kind"] == "rotary":
        phi, i0, i1 = _angles(c)
        cos, sin = phi.cos().float(), phi.sin().float()
        for x, out in ((s["q"], s["q_out"]), (s["k"], s["k_out"])):
            y = x.float().clone()
            a, b = x[..., i0].float(), x[..., i1].float()
            y[..., i0] = a * cos - b * sin
            y[..., i1] = a * sin + b * cos
            out.copy_(y)
        return [s["q_out"], s["k_out"]]
    if c["kind"] == "kv_cache":
        _to_cache(s["values"], s["exponents"], *_kv_views(c, s["kv"], c["n_tok"]), c["tok_offset"])
        x = s["values"].float() * _scale(s["exponents"])[..., None]
        k, v = _kv_views(c, s["back"], c["tokens"])
        k.copy_(x[:, 0])
        v.copy_(x[:, 1])
        return [s["back"]]
    x = s["values"].float() * _scale(s["exponents"])[..., None]
    if c["n_fresh"]:
        f = slice(c["fresh_begin"], c["fresh_begin"] + c["n_fresh"])
        x[:, 0, :, f], x[:, 1, :, f] = _kv_views(c, s["fresh"], c["n_fresh"])
    for b in range(c["B"]):
        p = s["q"][b].float() @ x[b, 0].transpose(1, 2)
        p *= 1.0 / math.sqrt(c["head_dim"])
        p -= p.amax(-1, keepdim=True)
        p.exp_()
        o = p @ x[b, 1] / p.sum(-1, keepdim=True)
        s["out"][b] = o.transpose(0, 1).reshape(c["n_q"], -1).to(_td(c))
    return [s["out"]]


def run(state):
    s = state
    if not own:
        return _run_plain(s)
    from paper_2509_04719_amd import _lib
    c = s["case"]
    B, heads, d = c["B"], c["heads"], c["head_dim"]
    code = _lib.DTYPE_CODE[c["dtype"]]
    if c["kind"] == "rotary":
        _lib.rotary(s["axes"], c["token_begin"], (s["q"], s["k"]), (s["q_out"], s["k_out"]))
        return [s["q_out"], s["k_out"]]
    if c["kind"] == "kv_cache":
        n, N, H = c["n_tok"], c["tokens"], heads * d
        _lib.kv_quantize(s["kv"], 2 * n * H, n, 0, s["cache"], c["tok_offset"], B, heads, n, d, code)
        _lib.kv_dequantize(s["cache"], 0, s["back"], 2 * N * H, N, 0, B, heads, N, d, code)
        return [s["back"]]
    nf = c["n_fresh"]
    _lib.attention_quantized(s["q"], s["cache"], s["fresh"], 2 * nf * heads * d, c["fresh_begin"], nf, B, heads,
                             c["n_q"], d, s["out"], code, workspace=s["workspace"])
    return [s["out"]]


# ---- the same in 64 bits -------------------------------------------------------

def _pow2(e):
    """2^e for whole numbers e, to the last bit (exp2 on the GPU is off by some)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _e4m3(x):
    """x (64 bits) rounded to the nearest e4m3 value, ties to even: steps of 2^(floor(log2 |x|) - 3), of 2^-9 below
    2^-6."""
    _, e = torch.frexp(x)
    step = _pow2((e - 4).clamp(min=-9))
    return torch.round(x / step) * step


def _quantized(x):
    """The values that x [..., d] (64 bits) has in the cache."""
    m, e = torch.frexp(x.abs().amax(-1, keepdim=True))          # max = m 2^e, 1/2 <= m < 1; 448 = 0.875 2^9
    e = torch.where(m > 0.875, e - 8, e - 9).clamp(min=-126)
    s = _pow2(e)
    return _e4m3(x / s) * s


def _cached(s):
    return s["values"].double() * _pow2(s["exponents"].long() - 127)[..., None]


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    B, heads, d = c["B"], c["heads"], c["head_dim"]
    if c["kind"] == "rotary":
        n = torch.arange(c["token_begin"], c["token_begin"] + c["n_tok"], device=DEV, dtype=torch.float64)
        cols, rows = c["cols"], c["rows"]
        row = torch.floor(n / cols)
        frame = torch.floor(row / rows)
        pos = (frame, (row - frame * rows + c["origin"]) * c["step"], (n - row * cols + c["origin"]) * c["step"])
        outs = []
        for x in (s["q"], s["k"]):
            parts, base = [], 0
            for p, ch in zip(pos, (c["ch_t"], c["ch_h"], c["ch_w"])):
                if ch == 0:
                    continue
                w = torch.exp(torch.arange(ch // 2, device=DEV, dtype=torch.float64) * (-2.0 / ch * math.log(c["theta"])))
                turn = torch.polar(torch.ones((), device=DEV, dtype=torch.float64), torch.outer(p, w))
                seg = x[..., base:base + ch].double()
                pairs = seg.unflatten(-1, (ch // 2, 2)) if c["interleaved"] else seg.unflatten(-1, (2, ch // 2)).transpose(-1, -2)
                z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
                parts.append((z if c["interleaved"] else z.transpose(-1, -2)).flatten(-2))
                base += ch
            parts.append(x[..., base:].double())
            outs.append(torch.cat(parts, -1))
        return outs
    if c["kind"] == "kv_cache":
        x = _cached(s)
        rows = slice(c["tok_offset"], c["tok_offset"] + c["n_tok"])
        k, v = _kv_views(c, s["kv"], c["n_tok"])
        x[:, 0, :, rows] = _quantized(k.double())
        x[:, 1, :, rows] = _quantized(v.double())
        return [torch.cat((x[:, 0].reshape(B, -1), x[:, 1].transpose(2, 3).reshape(B, -1)), 1)]
    x = _cached(s)
    if c["n_fresh"]:
        rows = slice(c["fresh_begin"], c["fresh_begin"] + c["n_fresh"])
        k, v = _kv_views(c, s["fresh"], c["n_fresh"])
        x[:, 0, :, rows], x[:, 1, :, rows] = k.double(), v.double()
    out = torch.empty((B, c["n_q"], heads, d), device=DEV, dtype=torch.float64)
    for b in range(B):
        for h in range(heads):
            z = s["q"][b, h].double() @ (x[b, 0, h].T.contiguous() / math.sqrt(d))
            out[b, :, h] = torch.exp(z - torch.logsumexp(z, -1, keepdim=True)) @ x[b, 1, h]
    return [out.flatten(2)]


# ---- what a pass cannot do without ----------------------------------------------

def work(case):
    c = case
    es = 4 if c["dtype"] == "f32" else 2
    B, heads, d = c["B"], c["heads"], c["head_dim"]
    if c["kind"] == "rotary":
        rows = 2 * B * heads * c["n_tok"]
        return {"bytes": 2.0 * rows * d * es, "flops": 3.0 * rows * (c["ch_t"] + c["ch_h"] + c["ch_w"])}
    if c["kind"] == "kv_cache":
        # the band in, its part of the cache out; the rest of the cache in, the buffer out
        n, N, rows = c["n_tok"], c["tokens"], 2 * B * heads
        return {"bytes": float(rows * (n * (d * es + d + 1) + (N - n) * (d + 1) + N * d * es)),
                "flops": 2.0 * rows * n * d + rows * N * d}
    n, N, nf, rows = c["n_q"], c["n_kv"], c["n_fresh"], B * heads
    return {"bytes": float(2 * rows * (n * d * es + nf * d * es + (N - nf) * (d + 1))),
            "flops": 4.0 * rows * n * N * d}
