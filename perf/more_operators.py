"""Norms around a block and products in 8-bit integers, as cases to be timed and compared.

Three kinds of calls, in the order in which a block makes them:

  norms      one pass between two blocks: the norm after the block that ends, its
             gate and the residual scale, the norm before the next one with its
             modulation
  product    a projection in 8-bit integers with a scale for each token and each
             output channel: plain, with GELU, added to the residual stream
             through a gate, or scattered into Q and the K/V buffer; its tokens
             come as codes, or as activations that are quantised in the call
  chain      both: the norms' result leaves as codes and goes into the product

`own` false: the operators in elementary torch operations, 32 bits throughout.
`own` true: the package's entry points.  Sizes are those of seeded_inputs/configs.py
(the tiny fp32 model, DiT-S/2 at 256px, DiT-XL/2 at 512, 1024 and 2048px) and
generic ones between them.
"""
import math

import torch

own = False

DEV = "cuda:0"


# ---- the cases ---------------------------------------------------------------

def _norms(name, B, n_tok, hidden, post, pre, affine, gate, modulate, has_y, has_out, residual_scale, pad, dtype):
    return {"name": name, "kind": "norms", "B": B, "n_tok": n_tok, "hidden": hidden, "post": post, "pre": pre,
            "affine": affine, "gate": gate, "modulate": modulate, "has_y": has_y, "has_out": has_out,
            "residual_scale": residual_scale, "pad": pad, "dtype": dtype}


def _product(name, B, n_tok, K, N, epilogue, codes, dtype, heads=0, tokens=0, tok_offset=0):
    return {"name": name, "kind": "product", "B": B, "n_tok": n_tok, "K": K, "N": N, "epilogue": epilogue,
            "codes": codes, "heads": heads, "tokens": tokens, "tok_offset": tok_offset, "dtype": dtype}


def _chain(name, B, n_tok, hidden, N, post, pre, epilogue, dtype):
    return {"name": name, "kind": "chain", "B": B, "n_tok": n_tok, "hidden": hidden, "K": hidden, "N": N,
            "post": post, "pre": pre, "affine": False, "gate": True, "modulate": True, "has_y": True,
            "has_out": True, "residual_scale": 1.0, "pad": 0, "epilogue": epilogue, "codes": True, "heads": 0,
            "tokens": 0, "tok_offset": 0, "dtype": dtype}


def listed():
    return [
        # the tiny fp32 model's half image: a call that is all launch and latency
        _norms("norms_tiny_f32", 1, 32, 128, "rms", "layer", False, True, True, True, True, 1.0, 0, "f32"),
        # an odd width, the block's output a slice of a wider buffer, learned weights, a scaled residual
        _norms("norms_odd_strided", 3, 171, 1021, "layer", "rms", True, True, False, True, True, 0.5, 64, "bf16"),
        # DiT-XL/2 at 1024px with guidance, the 40% band
        _norms("norms_xl1024_band40", 2, 26 * 64, 1152, "rms", "layer", False, True, True, True, True, 1.0, 0, "bf16"),
        # every row at 2048px
        _norms("norms_xl2048_all", 2, 128 * 128, 1152, "rms", "layer", True, True, True, True, True, 1.0, 0, "bf16"),
        # one token through the MLP's first product: its weights alone are read
        _product("product_one_token", 1, 1, 1152, 4608, "gelu", True, "bf16"),
        # odd sizes, fp32 activations and output (reference runs)
        _product("product_odd_f32", 1, 333, 1000, 777, "store", False, "f32"),
        # DiT-S/2 at 256px, its 40% band: Q, K and V of a small model
        _product("product_s2_256_qkv", 1, 96, 384, 1152, "qkv", True, "bf16", heads=6, tokens=256, tok_offset=80),
        # DiT-XL/2 at 1024px, the 40% band: the MLP's second product, from the activations, into the residual stream
        _product("product_xl1024_fc2", 2, 26 * 64, 4608, 1152, "residual", False, "bf16"),
        # 48 of 128 rows at 2048px: Q, K and V into the image's buffer
        _product("product_xl2048_qkv", 2, 48 * 128, 1152, 3456, "qkv", True, "bf16", heads=16, tokens=16384,
                 tok_offset=40 * 128),
        # every row at 2048px: the MLP's first product
        _product("product_xl2048_fc1", 2, 128 * 128, 1152, 4608, "gelu", True, "bf16"),
        # DiT-XL/2 at 512px, 12 of 32 rows: the norms into the MLP's first product
        _chain("chain_xl512_band12", 2, 12 * 32, 1152, 4608, "rms", "layer", "gelu", "bf16"),
        # DiT-XL/2 at 1024px, the 40% band: the norms into the projection of Q, K and V, kept together
        _chain("chain_xl1024_band40", 2, 26 * 64, 1152, 3456, "rms", "rms", "store", "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width: a multiple of 128, of 16, or any."""
    w = _log_int(rng, lo, hi)
    step = rng.choice((128, 128, 16, 1))
    return min(hi, max(step, w // step * step))


def draw(rng):
    """One more case of the listed kinds' ranges."""
    kind = rng.choice(("norms", "product", "product", "chain"))
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    B = rng.randint(1, 3)
    if kind == "norms":
        hidden = _width(rng, 32, 4608)
        rows = _log_int(rng, 1, max(1, 32768 * 1152 // (hidden * (2 if dtype == "f32" else 1))))
        B = min(B, rows)
        has_y = rng.random() < 0.85
        return {k: v for k, v in _norms(
            "", B, rows // B, hidden, rng.choice(("none", "layer", "rms", "rms")), rng.choice(("layer", "layer", "rms")),
            rng.random() < 0.5, rng.random() < 0.8, rng.random() < 0.8, has_y, not has_y or rng.random() < 0.85,
            rng.choice((1.0, 1.0, 0.5, 1.25)), rng.choice((0, 0, 8, 3)), dtype).items() if k != "name"}
    K = _width(rng, 128, 4608)
    if kind == "chain":
        N = _width(rng, 64, 4608)
        n_tok = _log_int(rng, 1, 8192) // B + 1
        c = _chain("", B, n_tok, K, N, rng.choice(("none", "layer", "rms")), rng.choice(("layer", "rms")),
                   rng.choice(("store", "gelu")), "bf16")
        del c["name"]
        return c
    epilogue = rng.choice(("store", "gelu", "residual", "qkv"))
    heads, tokens, off = 0, 0, 0
    if epilogue == "qkv":
        d = rng.choice((32, 64, 64, 72, 72, 80, 96, 128))
        heads = rng.randint(1, 1152 // d)
        N = 3 * heads * d
    else:
        N = _width(rng, 64, 4608)
    most = 32768 * 1152 * 4608 // (K * N)
    M = min(_log_int(rng, 1, 32768), most, 32768 * 1152 // max(K, N) * 2)
    n_tok = max(1, M // B)
    if epilogue == "qkv":
        tokens = n_tok + rng.choice((0, 1, _log_int(rng, 1, 4096)))
        off = rng.randint(0, tokens - n_tok)
    c = _product("", B, n_tok, K, N, epilogue, rng.random() < 0.5, dtype, heads, tokens, off)
    del c["name"]
    return c


# ---- inputs --------------------------------------------------------------------

def _td(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 31)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _quantize(x):
    """Codes and scales of the rows of x (32 bits): 127 for a row's largest magnitude, to nearest, ties to even."""
    top = x.abs().amax(-1)
    full = torch.full_like(top, 127.0)
    r = torch.where(top > 0, full / top, torch.zeros_like(top))
    return torch.round(x * r[:, None]), top / full


def _codes(x):
    """The same as held: int8 rows a multiple of 16 bytes apart."""
    q, s = _quantize(x)
    held = torch.zeros((q.shape[0], -(-q.shape[1] // 16) * 16), dtype=torch.int8, device=DEV)
    held[:, :q.shape[1]] = q.to(torch.int8)
    return held[:, :q.shape[1]], s


def prepare(case, seed):
    c = case
    g = _gen(seed)
    s = {"case": c}
    rows, td = c["B"] * c["n_tok"], _td(c)
    if c["kind"] != "product":
        H = c["hidden"]
        # the residual stream: some channels far from zero, some tokens larger than others
        s["h"] = _randn(g, rows, H) * torch.exp(0.5 * _randn(g, rows, 1)) + 3.0 * _randn(g, 1, H)
        s["y"] = None
        if c["has_y"]:
            wide = (_randn(g, rows, H + c["pad"]) * torch.exp(0.7 * _randn(g, 1, H + c["pad"]))).to(td)
            s["y"] = wide[:, c["pad"]:]
        # the adaLN vectors, as the conditioning leaves them: gate, shift and scale next to each other
        mod = 0.3 * _randn(g, c["B"], 3, H)
        s["gate"] = mod[:, 0] if c["gate"] else None
        s["shift"], s["scale"] = (mod[:, 1], mod[:, 2]) if c["modulate"] else (None, None)
        for p in ("post", "pre"):
            s[p + "_w"] = 1.0 + 0.2 * _randn(g, H) if c["affine"] else None
        s["h_out"] = torch.empty_like(s["h"]) if c["has_y"] else None
        s["out"] = torch.empty((rows, H), dtype=td, device=DEV) if c["has_out"] and c["kind"] == "norms" else None
    if c["kind"] != "norms":
        K, N = c["K"], c["N"]
        s["w"], s["w_s"] = _codes(_randn(g, N, K) * (0.02 * torch.exp(0.3 * _randn(g, N, 1))))
        s["bias"] = 0.1 * _randn(g, N)
        if c["kind"] == "product":
            x = (_randn(g, rows, K) * torch.exp(0.7 * _randn(g, 1, K)) * torch.exp(0.5 * _randn(g, rows, 1))).to(td)
            if c["codes"]:
                s["a"], s["a_s"] = _codes(x.float())
            else:
                s["x"] = x
        if c["kind"] == "chain" or not c["codes"]:
            s["a"] = torch.zeros((rows, -(-K // 16) * 16), dtype=torch.int8, device=DEV)[:, :K]
            s["a_s"] = torch.zeros(rows, device=DEV)
        if c["epilogue"] == "qkv":
            hidden = N // 3
            s["q"] = torch.empty((c["B"], c["heads"], c["n_tok"], hidden // c["heads"]), dtype=td, device=DEV)
            s["kv"] = torch.empty((c["B"], 2 * c["tokens"] * hidden), dtype=td, device=DEV).fill_(0.25)
        elif c["epilogue"] == "residual":
            s["res"] = _randn(g, rows, N)
            s["gate"] = 0.3 * _randn(g, c["B"], N)
            s["prod"] = torch.empty((rows, N), device=DEV)
        else:
            s["prod"] = torch.empty((rows, N), dtype=td, device=DEV)
    if own:
        from paper_2509_04719_amd import _lib
        if c["kind"] != "product":
            s["n_post"] = _lib.norm(c["post"], 1e-6, s["post_w"])
            s["n_pre"] = _lib.norm(c["pre"], 1e-6, s["pre_w"])
        if c["kind"] != "norms":
            s["W8"] = _lib.int8_rows(s["w"], s["w_s"])
            s["A8"] = _lib.int8_rows(s["a"], s["a_s"])
            need = _lib.linear_quantized_workspace_bytes(rows, c["N"], c["K"])
            s["workspace"] = torch.empty(need, dtype=torch.uint8, device=DEV) if need else None
    return s


# ---- one pass ------------------------------------------------------------------

def _norm(x, kind, w):
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    if kind != "none":
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)
    return x if w is None else x * w


def _per_token(c, v):
    return v.repeat_interleave(c["n_tok"], 0)


def _plain_norms(s):
    """The residual stream and the next block's input, 32 bits."""
    c = s["case"]
    h = s["h"] * c["residual_scale"]
    if c["has_y"]:
        z = _norm(s["y"].float(), c["post"], s["post_w"])
        h = h + (z if s["gate"] is None else _per_token(c, s["gate"]) * z)
    if not c["has_out"]:
        return h, None
    u = _norm(h, c["pre"], s["pre_w"])
    if c["modulate"]:
        u = u * (1.0 + _per_token(c, s["scale"])) + _per_token(c, s["shift"])
    return h, u


def _plain_product(s, q, scales):
    """codes q and scales of the tokens -> the outputs."""
    c = s["case"]
    y = q.float() @ s["w"].float().t()
    y = y * scales[:, None] * s["w_s"] + s["bias"]
    if c["epilogue"] == "gelu":
        y = 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))
    if c["epilogue"] == "residual":
        s["prod"].copy_(s["res"] + _per_token(c, s["gate"]) * y)
        return [s["prod"]]
    if c["epilogue"] != "qkv":
        s["prod"].copy_(y)
        return [s["prod"]]
    B, n, heads, N = c["B"], c["n_tok"], c["heads"], c["tokens"]
    qkv = y.view(B, n, 3, heads, -1).permute(2, 0, 3, 1, 4)
    s["q"].copy_(qkv[0])
    k, v = s["kv"].view(B, 2, -1).unbind(1)
    band = slice(c["tok_offset"], c["tok_offset"] + n)
    k.view(B, heads, N, -1)[:, :, band] = qkv[1].to(k.dtype)
    v.view(B, heads, -1, N)[..., band] = qkv[2].transpose(2, 3).to(v.dtype)
    return [s["q"], s["kv"]]


def _run_plain(s):
    c = s["case"]
    if c["kind"] == "product":
        return _plain_product(s, s["a"], s["a_s"]) if c["codes"] else _plain_product(s, *_quantize(s["x"].float()))
    h, u = _plain_norms(s)
    outs = []
    if s["h_out"] is not None:
        s["h_out"].copy_(h)
        outs.append(s["h_out"])
    if c["kind"] == "chain":
        return outs + _plain_product(s, *_quantize(u))
    if s["out"] is not None:
        s["out"].copy_(u)
        outs.append(s["out"])
    return outs


def _own_product(lib, s):
    c = s["case"]
    if c["epilogue"] == "qkv":
        lib.qkv_projection_quantized(s["A8"], s["W8"], s["bias"], s["q"], s["kv"], c["tokens"], c["tok_offset"],
                                workspace=s["workspace"])
        return [s["q"], s["kv"]]
    if c["epilogue"] == "residual":
        s["prod"].copy_(s["res"])
        lib.linear_quantized(s["A8"], s["W8"], s["bias"], lib.EPI_RESIDUAL, s["prod"], gate=s["gate"],
                        rows_per_batch=c["n_tok"], workspace=s["workspace"])
    else:
        lib.linear_quantized(s["A8"], s["W8"], s["bias"], lib.EPI_GELU if c["epilogue"] == "gelu" else lib.EPI_STORE,
                        s["prod"], workspace=s["workspace"])
    return [s["prod"]]


def run(state):
    s = state
    if not own:
        return _run_plain(s)
    from paper_2509_04719_amd import _lib
    c = s["case"]
    if c["kind"] == "product":
        if not c["codes"]:
            _lib.quantize_rows(s["x"], s["A8"])
        return _own_product(_lib, s)
    out = s["A8"] if c["kind"] == "chain" else s["out"]
    _lib.block_norms(s["h"], s["y"], s["h_out"], out, post=s["n_post"], pre=s["n_pre"], gate=s["gate"],
                     shift=s["shift"], scale=s["scale"], rows_per_batch=c["n_tok"],
                     residual_scale=c["residual_scale"])
    outs = [s["h_out"]] if s["h_out"] is not None else []
    if c["kind"] == "chain":
        return outs + _own_product(_lib, s)
    return outs + ([out] if out is not None else [])


# ---- the same in 64 bits -------------------------------------------------------

def _exact_norm(x, kind, w):
    """(x - center) / sqrt(mean square of it + eps), row by row."""
    center = torch.sum(x, 1) / x.shape[1] if kind == "layer" else torch.zeros(x.shape[0], dtype=x.dtype, device=DEV)
    if kind != "none":
        x = x - center[:, None]
        x = x / torch.sqrt(torch.sum(x ** 2, 1) / x.shape[1] + 1e-6)[:, None]
    return x if w is None else x * w.double()


def _exact_codes(x):
    """The codes by their definition (127 / max |x| and x times it are rounded to 32 bits, then to the nearest whole
    number), and what one of them stands for."""
    top = torch.amax(torch.abs(x), 1)
    some = torch.where(top > 0, top, torch.ones_like(top))
    r = (127.0 / some).float().double()
    return torch.round((x * r[:, None]).float().double()), top / 127.0


def _exact_product(s, n, unit):
    c = s["case"]
    B, N = c["B"], c["N"]
    w = s["w"].double() * s["w_s"].double()[:, None]
    y = torch.addmm(s["bias"].double(), n * unit[:, None], w.t().contiguous())
    if c["epilogue"] == "gelu":
        u = math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3)
        return [y / (1.0 + torch.exp(-2.0 * u))]
    if c["epilogue"] == "residual":
        return [(s["res"].double().view(B, -1, N) + s["gate"].double()[:, None] * y.view(B, -1, N)).view(-1, N)]
    if c["epilogue"] == "store":
        return [y]
    heads, n_tok, tokens, off = c["heads"], c["n_tok"], c["tokens"], c["tok_offset"]
    d = N // 3 // heads
    q, k, v = (y[:, i * heads * d:(i + 1) * heads * d].view(B, n_tok, heads, d) for i in range(3))
    buf = s["kv"].double()
    kk, vv = buf[:, :tokens * heads * d].view(B, heads, tokens, d), buf[:, tokens * heads * d:].view(B, heads, d, tokens)
    for h in range(heads):
        kk[:, h, off:off + n_tok] = k[:, :, h]
        for b in range(B):
            vv[b, h, :, off:off + n_tok] = v[b, :, h].t()
    return [q.permute(0, 2, 1, 3).contiguous(), buf]


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["kind"] == "product":
        return _exact_product(s, s["a"].double(), s["a_s"].double()) if c["codes"] else \
            _exact_product(s, *_exact_codes(s["x"].double()))
    B, n, H = c["B"], c["n_tok"], c["hidden"]
    h = c["residual_scale"] * s["h"].double()
    if c["has_y"]:
        z = _exact_norm(s["y"].double(), c["post"], s["post_w"]).view(B, n, H)
        g = torch.ones((B, H), dtype=torch.float64, device=DEV) if s["gate"] is None else s["gate"].double()
        h = h + (z * g[:, None]).view(B * n, H)
    outs = [h] if s["h_out"] is not None else []
    if not c["has_out"]:
        return outs
    u = _exact_norm(h, c["pre"], s["pre_w"])
    if c["modulate"]:
        u = (u.view(B, n, H) * (s["scale"].double() + 1.0)[:, None] + s["shift"].double()[:, None]).view(B * n, H)
    return outs + (_exact_product(s, *_exact_codes(u)) if c["kind"] == "chain" else [u])


# ---- what a pass cannot do without ----------------------------------------------

def work(case):
    c = case
    es = 4 if c["dtype"] == "f32" else 2
    rows = c["B"] * c["n_tok"]
    bytes_, flops = 0.0, 0.0
    if c["kind"] != "product":
        H = c["hidden"]
        # the stream in and (where a block ended) out, the block's output in, the next one's input out
        bytes_ += rows * H * (4.0 + (4.0 + es if c["has_y"] else 0.0))
        if c["has_out"] and c["kind"] == "norms":
            bytes_ += rows * H * es
        flops += rows * H * ((8.0 if c["has_y"] else 0.0) + (8.0 if c["has_out"] else 0.0))
    if c["kind"] != "norms":
        K, N = c["K"], c["N"]
        # (the chain's codes go from one call to the next)
        bytes_ += N * (K + 8.0) + rows * N * (8.0 if c["epilogue"] == "residual" else es)
        if c["kind"] == "product":
            bytes_ += rows * (K + 4.0 if c["codes"] else K * es)
        flops += 2.0 * rows * N * K
    return {"bytes": float(bytes_), "flops": float(flops)}
