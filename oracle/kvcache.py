"""Rotary positions, the 8-bit K/V cache and attention over it, in float64."""
import numpy as np


def rotary(x, token_begin, channels, extent, origin, step, theta, interleaved):
    """x [B, heads, n, d] -> rotated; token n = (f * rows + r) * cols + c."""
    out = x.astype(np.float64).copy()
    n = token_begin + np.arange(x.shape[2])
    _, R, Cc = extent
    index = (n // (R * Cc), (n // Cc) % R, n % Cc)
    base = 0
    for a in range(3):
        ch = channels[a]
        for i in range(ch // 2):
            phi = (index[a] + origin[a]) * step[a] * theta ** (-2.0 * i / ch)
            p, q = (base + 2 * i, base + 2 * i + 1) if interleaved else (base + i, base + ch // 2 + i)
            u, v = x[..., p].astype(np.float64), x[..., q].astype(np.float64)
            out[..., p] = u * np.cos(phi) - v * np.sin(phi)
            out[..., q] = u * np.sin(phi) + v * np.cos(phi)
        base += ch
    return out


def e4m3_table():
    """The 256 values of an e4m3 byte: sign, 4 exponent bits (bias 7), 3 of mantissa; 0x7f and 0xff are NaN."""
    b = np.arange(256)
    e, m = (b >> 3) & 15, b & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v[(b & 127) == 127] = np.nan
    return np.where(b >= 128, -v, v)


def to_e4m3(x):
    """Bytes of the nearest e4m3 values (|x| <= 448), ties to the even mantissa; not finite: NaN."""
    tab = e4m3_table()[:127]                       # 0 .. 448, rising
    mid = 0.5 * (tab[1:] + tab[:-1])
    a = np.abs(np.where(np.isfinite(x), x, 0.0))
    lo = np.searchsorted(mid, a, side="left")      # a tie goes to the lower one
    tie = (lo < 126) & (a == mid[np.minimum(lo, 125)])
    code = lo + (tie & (lo % 2 == 1))              # an odd mantissa: the upper one is even
    code = np.where(np.isfinite(x), code, 127)
    return (code | np.where(np.signbit(x) & np.isfinite(x), 128, 0)).astype(np.uint8)


def quantize(x):
    """x [..., d] -> (e4m3 bytes [..., d], E8M0 bytes [...])."""
    x = x.astype(np.float64)
    fin = np.isfinite(x)
    amax = np.max(np.where(fin, np.abs(x), 0.0), axis=-1)
    e = np.full(amax.shape, -126)
    pos = amax > 0
    m, k = np.frexp(amax[pos])                     # amax = m 2^k, 1/2 <= m < 1; 448 = 0.875 2^9
    e[pos] = np.maximum(np.where(m > 0.875, k - 8, k - 9), -126)
    top = 1.875 * 2.0 ** 127
    y = np.where(fin, np.clip(x, -top, top), x) / 2.0 ** e[..., None].astype(np.float64)
    return to_e4m3(y), (e + 127).astype(np.uint8)


def dequantize(values, exponents):
    return e4m3_table()[values] * 2.0 ** (exponents.astype(np.float64) - 127.0)[..., None]


def attention(q, k, v, absolute=False):
    """q [.., n_q, d], k and v [.., n, d] -> softmax(q k^T / sqrt d) v; absolute: also the sums of p |v|."""
    s = q.astype(np.float64) @ np.swapaxes(k.astype(np.float64), -1, -2) / np.sqrt(q.shape[-1])
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    return (p @ v, p @ np.abs(v)) if absolute else p @ v


def to_buffer(k, v):
    """k, v [B, heads, n, d] -> [B, 2 n heads d]: K [heads][n][d], then V^T [heads][d][n]."""
    B = k.shape[0]
    return np.concatenate([k.reshape(B, -1), np.swapaxes(v, -1, -2).reshape(B, -1)], axis=1)


def from_buffer(buf, heads, n, d):
    B = buf.shape[0]
    k, vt = buf.reshape(B, 2, -1)[:, 0], buf.reshape(B, 2, -1)[:, 1]
    return k.reshape(B, heads, n, d), np.swapaxes(vt.reshape(B, heads, d, n), -1, -2)
