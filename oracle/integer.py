"""Norms around a block in float64; rows in 8-bit integers with a scale each, and their products."""
import numpy as np


def norm(x, kind, eps=1e-6, weight=None, bias=None):
    """x [rows, hidden]: (x - mean) / sqrt(var + eps), x / sqrt(mean x^2 + eps) or x; times weight plus bias."""
    x = np.asarray(x, dtype=np.float64)
    if kind == "layer":
        x = (x - x.mean(1, keepdims=True)) / np.sqrt(x.var(1, keepdims=True) + eps)
    elif kind == "rms":
        x = x / np.sqrt((x * x).mean(1, keepdims=True) + eps)
    if weight is not None:
        x = x * weight
    return x if bias is None else x + bias


def rows_of(v, rows, rows_per_batch, default):
    """Row r of the result is row r / rows_per_batch of v."""
    return default if v is None else np.asarray(v, dtype=np.float64)[np.arange(rows) // rows_per_batch]


def block_norms(h, y, post, pre, gate=None, shift=None, scale=None, rows_per_batch=1, residual_scale=1.0):
    """(h', u); post and pre are arguments of norm() after x."""
    n = h.shape[0]
    h1 = residual_scale * np.asarray(h, dtype=np.float64)
    if y is not None:
        h1 = h1 + rows_of(gate, n, rows_per_batch, 1.0) * norm(y, *post)
    u = norm(h1, *pre) * (1.0 + rows_of(scale, n, rows_per_batch, 0.0)) + rows_of(shift, n, rows_per_batch, 0.0)
    return h1, u


def quantize_rows(x):
    """float32 [rows, cols] -> int8 codes, float32 scales: code = x * (127 / max |x|), quotient and product
    rounded to 32 bits (of 2^64 x below 2^-64), to nearest, ties to even."""
    x = np.asarray(x, dtype=np.float32)
    f = np.float32
    codes, scales = np.zeros(x.shape, np.int8), np.zeros(x.shape[0], f)
    for r, row in enumerate(x):
        if not np.isfinite(row).all():
            scales[r] = np.nan
            continue
        top = np.abs(row).max()
        if top == 0:
            continue
        up = f(2.0 ** 64) if top < f(2.0 ** -64) else f(1)
        codes[r] = np.rint((row * up) * (f(127) / (top * up))).astype(np.int8)
        scales[r] = top / f(127)
    return codes, scales


def product(a, sa, w, sw, bias=None):
    """a [M, K], w [N, K] int8 -> float64 [M, N]; exact sums."""
    s = a.astype(np.float64) @ w.astype(np.float64).T       # |sum| < 2^31: exact
    y = s * np.asarray(sa, np.float64)[:, None] * np.asarray(sw, np.float64)
    return y if bias is None else y + bias


def gelu_tanh(y):
    return 0.5 * y * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (y + 0.044715 * y ** 3)))


def qkv(y, B, heads, kv, kv_tokens, tok_offset):
    """y [B n, 3 H] -> Q [B, heads, n, d]; K and V of the n tokens into kv [B, 2 kv_tokens H] (K [heads][kv_tokens][d],
    then V^T [heads][d][kv_tokens])."""
    n, H = y.shape[0] // B, y.shape[1] // 3
    q, k, v = (y[:, i * H:(i + 1) * H].reshape(B, n, heads, H // heads).transpose(0, 2, 1, 3) for i in range(3))
    kv = np.array(kv, dtype=np.float64)
    kb, vb = kv[:, :kv_tokens * H].reshape(B, heads, kv_tokens, -1), kv[:, kv_tokens * H:2 * kv_tokens * H].reshape(B, heads, -1, kv_tokens)
    kb[:, :, tok_offset:tok_offset + n] = k
    vb[..., tok_offset:tok_offset + n] = v.transpose(0, 1, 3, 2)
    kv[:, :kv_tokens * H], kv[:, kv_tokens * H:2 * kv_tokens * H] = kb.reshape(B, -1), vb.reshape(B, -1)
    return q, kv
