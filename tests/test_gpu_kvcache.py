"""The 8-bit K/V cache against the oracle: bytes equal when written, values equal when read back."""
import numpy as np
import pytest
import torch

from oracle import kvcache as ok
from tests._gpu_util import DEV, code, rounded, to_dev, to_host

pytestmark = pytest.mark.gpu


def _kv(rng, B, heads, n, d, dtype):
    """K and V over many magnitudes, some exactly between two e4m3 values."""
    x = [rng.standard_normal((B, heads, n, d)) * 2.0 ** rng.integers(-6, 6, (B, heads, n, 1)) for _ in range(2)]
    for a in x:
        a[..., ::5] *= 2.0 ** -9
        a[..., 1::7] = np.round(a[..., 1::7] * 16) / 16
    return [rounded(a, dtype) for a in x]


def _empty(B, heads, tokens, d, pad=0):
    v = torch.full((B, 2 * heads * tokens * d + pad), 0x55, dtype=torch.uint8, device=DEV)
    e = torch.full((B, 2 * heads * tokens + pad), 0x33, dtype=torch.uint8, device=DEV)
    return (v[:, :2 * heads * tokens * d].unflatten(1, (2, heads, tokens, d)),
            e[:, :2 * heads * tokens].unflatten(1, (2, heads, tokens)))


# tokens of the cache, first, count; tokens of the buffer, first
BANDS = [(1, 0, 1, 1, 0), (64, 16, 32, 32, 0), (64, 0, 64, 64, 0), (77, 5, 71, 71, 0), (130, 64, 1, 9, 8), (200, 61, 67, 100, 32),
         (96, 24, 40, 43, 3)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 72, 80, 96, 128])
@pytest.mark.parametrize("N,off,n,T,kv_off", BANDS)
def test_write_and_read_back(orch_lib, dtype, d, N, off, n, T, kv_off):
    B, heads = 2, 3
    rng = np.random.default_rng(d + N + n)
    k, v = _kv(rng, B, heads, T, d, dtype)
    buf = to_dev(ok.to_buffer(k, v), dtype)
    pad = 48                                            # branches that do not follow each other
    values, exps = _empty(B, heads, N, d, pad)
    cache = orch_lib.quantized_kv(values, exps)
    orch_lib.kv_quantize(buf, 2 * T * heads * d, T, kv_off, cache, off, B, heads, n, d, code(dtype))
    torch.cuda.synchronize()
    wv, we = np.full((B, 2, heads, N, d), 0x55, np.uint8), np.full((B, 2, heads, N), 0x33, np.uint8)
    for i, x in enumerate((k, v)):
        wv[:, i, :, off:off + n], we[:, i, :, off:off + n] = ok.quantize(x[:, :, kv_off:kv_off + n])
    np.testing.assert_array_equal(exps.cpu().numpy(), we)
    np.testing.assert_array_equal(values.cpu().numpy(), wv)     # (and what lies outside the band as it was)
    assert torch.all(values.as_strided((B, pad), (values.stride(0), 1), 2 * heads * N * d) == 0x55)
    # back into a buffer of both other extents, at another offset
    T2, off2 = n + 13, 8 if n % 8 == 0 else 5
    back = torch.full((B, 2 * T2 * heads * d + 16), 7.0, dtype=buf.dtype, device=DEV)
    orch_lib.kv_dequantize(cache, off, back, 2 * T2 * heads * d + 16, T2, off2, B, heads, n, d, code(dtype))
    got = to_host(back)
    assert (got[:, -16:] == 7).all()
    gk, gv = ok.from_buffer(got[:, :-16], heads, T2, d)
    for g, i in ((gk, 0), (gv, 1)):
        want = np.full((B, heads, T2, d), 7.0)
        want[:, :, off2:off2 + n] = ok.dequantize(wv[:, i, :, off:off + n], we[:, i, :, off:off + n])
        np.testing.assert_array_equal(g, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_edges_of_the_types(orch_lib, dtype):
    """Zeros, the types' largest and smallest numbers, infinities and NaN, and 448 and its neighbours as the largest."""
    heads, d = 1, 32
    rows = [np.zeros(d), np.full(d, 2.0 ** -133), np.full(d, 3.3895e38), np.full(d, -1.99 * 2.0 ** 127),
            np.linspace(-448, 448, d), np.linspace(-464, 464, d), np.linspace(-1, 1, d) * 2.0 ** -126, np.full(d, 1e-30)]
    for bad in (np.inf, -np.inf, np.nan):
        r = np.linspace(0.1, 2, d)
        r[3], r[4] = bad, -bad
        rows.append(r)
    rows.append(np.full(d, np.nan))
    x = np.stack(rows)
    with np.errstate(all="ignore"):
        x = x.astype(np.float32)
    xt = torch.from_numpy(x).to(DEV)
    xt = xt if dtype == "f32" else xt.bfloat16()
    x = xt.double().cpu().numpy()
    n = len(rows)
    buf = torch.cat((xt.reshape(-1), xt.T.reshape(-1))).contiguous()
    values, exps = _empty(1, heads, n, d)
    cache = orch_lib.quantized_kv(values, exps)
    orch_lib.kv_quantize(buf, 0, n, 0, cache, 0, 1, heads, n, d, code(dtype))
    back = torch.empty_like(buf)
    orch_lib.kv_dequantize(cache, 0, back, 0, n, 0, 1, heads, n, d, code(dtype))
    torch.cuda.synchronize()
    wv, we = ok.quantize(x)
    want = ok.dequantize(wv, we)
    for i in range(2):
        np.testing.assert_array_equal(exps[0, i, 0].cpu().numpy(), we)
        got = values[0, i, 0].cpu().numpy()
        nan = np.isnan(want)
        np.testing.assert_array_equal(got[~nan], wv[~nan])
        assert ((got[nan] & 127) == 127).all()
    # bf16 has no number below 2^-133: the nearest
    want = torch.from_numpy(want).float().to(buf.dtype).double().numpy()
    k, v = ok.from_buffer(to_host(back)[None], heads, n, d)
    np.testing.assert_array_equal(k[0, 0], want)
    np.testing.assert_array_equal(v[0, 0], want)
    assert np.isfinite(want[:8]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bands_in_any_order_are_the_whole(orch_lib, dtype):
    """A token's bytes depend on the token alone: bands cut anywhere and written in any order give the bytes of one call."""
    B, heads, N, d = 1, 4, 111, 72
    rng = np.random.default_rng(3)
    buf = to_dev(ok.to_buffer(*_kv(rng, B, heads, N, d, dtype)), dtype)
    va, ea = _empty(B, heads, N, d)
    vb, eb = _empty(B, heads, N, d)
    orch_lib.kv_quantize(buf, 0, N, 0, orch_lib.quantized_kv(va, ea), 0, B, heads, N, d, code(dtype))
    c = orch_lib.quantized_kv(vb, eb)
    for lo, hi in ((50, 111), (0, 1), (9, 50), (1, 9)):
        orch_lib.kv_quantize(buf, 0, N, lo, c, lo, B, heads, hi - lo, d, code(dtype))
    orch_lib.kv_quantize(buf, 0, N, 3, c, 3, B, heads, 0, d, code(dtype))      # no tokens
    assert torch.equal(va, vb) and torch.equal(ea, eb)


def test_a_large_cache(orch_lib):
    """More than 2^32 bytes from the first value to the last: the last head's last tokens."""
    B, heads, d, N = 2, 16, 128, 1 << 20
    values = torch.empty((B, 2, heads, N, d), dtype=torch.uint8, device=DEV)
    exps = torch.empty((B, 2, heads, N), dtype=torch.uint8, device=DEV)
    assert values.numel() > 2 ** 32
    n, rng = 40, np.random.default_rng(1)
    k, v = _kv(rng, B, heads, n, d, "bf16")
    buf = to_dev(ok.to_buffer(k, v), "bf16")
    cache = orch_lib.quantized_kv(values, exps)
    orch_lib.kv_quantize(buf, 2 * n * heads * d, n, 0, cache, N - n, B, heads, n, d, 1)
    back = torch.empty_like(buf)
    orch_lib.kv_dequantize(cache, N - n, back, 2 * n * heads * d, n, 0, B, heads, n, d, 1)
    gk, gv = ok.from_buffer(to_host(back), heads, n, d)
    for i, (g, x) in enumerate(((gk, k), (gv, v))):
        wv, we = ok.quantize(x)
        np.testing.assert_array_equal(values[:, i, :, N - n:].cpu().numpy(), wv)
        np.testing.assert_array_equal(exps[:, i, :, N - n:].cpu().numpy(), we)
        np.testing.assert_array_equal(g, ok.dequantize(wv, we))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_branch_in_one_record(orch_lib, dtype):
    """Values and exponents of a branch one behind the other, as a peer would get them: the bytes and results of a cache in
    two tensors, nothing between the records touched."""
    B, heads, d, N, n = 3, 4, 72, 75, 33
    rng = np.random.default_rng(2)
    buf = to_dev(ok.to_buffer(*_kv(rng, B, heads, N, d, dtype)), dtype)
    v, e = 2 * heads * N * d, 2 * heads * N
    rec = torch.full((B, (v + e + 15) // 16 * 16 + 32), 0x55, dtype=torch.uint8, device=DEV)
    pairs = [_empty(B, heads, N, d), (rec[:, :v].unflatten(1, (2, heads, N, d)), rec[:, v:v + e].unflatten(1, (2, heads, N)))]
    q = to_dev(rng.standard_normal((B, heads, n, d)), dtype)
    results = []
    for values, exps in pairs:
        cache = orch_lib.quantized_kv(values, exps)
        orch_lib.kv_quantize(buf, 2 * N * heads * d, N, 0, cache, 0, B, heads, N, d, code(dtype))
        back = torch.empty_like(buf)
        orch_lib.kv_dequantize(cache, 0, back, 2 * N * heads * d, N, 0, B, heads, N, d, code(dtype))
        out = torch.empty((B, n, heads * d), dtype=buf.dtype, device=DEV)
        orch_lib.attention_quantized(q, cache, None, 0, 0, 0, B, heads, n, d, out, code(dtype))
        results.append((values.clone(), exps.clone(), back, out))
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert torch.all(rec[:, v + e:] == 0x55)
