"""Rows in 8-bit integers and their products against the oracle."""
import numpy as np
import pytest
import torch

from oracle import integer as oi
from tests._gpu_util import DEV, code, rounded, to_dev, to_host

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": U, "bf16": 2.0 ** -8}
FORMS = range(7)


@pytest.fixture(params=FORMS)
def form(request, monkeypatch):
    monkeypatch.setenv("ORCH_INT8_TILE", str(request.param))
    return request.param


# ---- the quantiser --------------------------------------------------------------

def _rows(rng, rows, cols, dtype):
    x = rng.standard_normal((rows, cols)) * 2.0 ** rng.integers(-8, 8, (rows, 1))
    x[:, ::5] = np.round(x[:, ::5] * 16) / 16           # ties
    return rounded(x, dtype)


def _quantize(lib, x, dtype, pad=0, gap=0):
    rows, cols = x.shape
    xd = torch.cat((torch.full((rows, pad), 1e9, device=DEV).to(to_dev(x, dtype).dtype), to_dev(x, dtype)), 1)[:, pad:]
    C = -(-cols // 16) * 16 + gap
    values, scales = torch.full((rows, C), 85, dtype=torch.int8, device=DEV), torch.full((rows + 3,), 6.0, device=DEV)
    lib.quantize_rows(xd, lib.int8_rows(values[:, :cols], scales[:rows]))
    torch.cuda.synchronize()
    assert torch.all(values[:, cols:] == 85) and torch.all(scales[rows:] == 6.0)
    return values[:, :cols].cpu().numpy(), scales[:rows].cpu().numpy()


COLS = [1, 7, 8, 100, 128, 129, 1000, 1024, 1026, 1152, 1280, 1288, 4608, 4616, 18432, 18440, 20001]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", COLS)
def test_codes_are_exact(orch_lib, dtype, cols):
    rng = np.random.default_rng(cols)
    for rows, pad, gap in ((1, 0, 0), (9, 0, 16), (13, 8, 0), (6, 3, 32)):
        x = _rows(rng, rows, cols, dtype)
        q, s = _quantize(orch_lib, x, dtype, pad, gap)
        wq, ws = oi.quantize_rows(x)
        np.testing.assert_array_equal(s, ws)
        np.testing.assert_array_equal(q, wq)


def test_longest_rows(orch_lib):
    x = _rows(np.random.default_rng(0), 2, 131071, "bf16")
    q, s = _quantize(orch_lib, x, "bf16")
    wq, ws = oi.quantize_rows(x)
    np.testing.assert_array_equal(q, wq)
    np.testing.assert_array_equal(s, ws)


@pytest.mark.parametrize("cols", [64, 65, 5000, 20000])
def test_extreme_rows(orch_lib, cols):
    """Zeros, subnormals, the largest magnitudes, and what is not finite."""
    rng = np.random.default_rng(1)
    x = rng.standard_normal((9, cols)).astype(np.float32)
    x[0], x[1], x[2] = 0.0, x[1] * np.float32(2.0 ** -140), x[2] * np.float32(2.0 ** -66)
    x[3] *= np.float32(2.0 ** 124)
    x[4, cols // 2], x[5, 0], x[6, cols - 1] = np.nan, np.inf, -np.inf
    x[7], x[7, 3] = 0.0, np.float32(2.0 ** -149)
    q, s = _quantize(orch_lib, x, "f32")
    wq, ws = oi.quantize_rows(x)
    np.testing.assert_array_equal(s, ws)
    np.testing.assert_array_equal(q, wq)


# ---- products -------------------------------------------------------------------

def _codes(rng, rows, cols, gap=0, garbage=True):
    """int8 rows over the whole range, -128 among it, and what lies behind them must not matter."""
    v = rng.integers(-128, 128, (rows, cols), dtype=np.int8)
    C = -(-cols // 16) * 16 + gap
    held = np.full((rows, C), 127, np.int8)
    held[:, :cols] = v
    return v, torch.from_numpy(held).to(DEV)[:, :cols]


def _operands(lib, rng, M, K, N, gap=0):
    a, ad = _codes(rng, M, K, gap)
    w, wd = _codes(rng, N, K, gap and 48)
    sa, sw = (np.exp(rng.standard_normal(n)).astype(np.float32) / np.float32(100 * np.sqrt(K)) for n in (M, N))
    bias = rng.standard_normal(N).astype(np.float32)
    A, W = lib.int8_rows(ad, to_dev(sa)), lib.int8_rows(wd, to_dev(sw))
    return A, W, bias, oi.product(a, sa, w, sw), a, sa, w, sw


def _check(got, want, off, dtype):
    over = np.abs(got - want) - (HALF[dtype] * np.abs(want) + off * (1 + HALF[dtype]))
    assert (over <= 0).all(), (float(over.max()), np.unravel_index(over.argmax(), over.shape))


def _gelu_off(y, off):
    """y off by `off` moves the result by 1.13 of it at most; its exponent is off by four roundings of
    itself, exp2 and the sum by three, the reciprocal and product by four (2^-22)."""
    z = 2 * np.sqrt(2 / np.pi) * np.abs(y + 0.044715 * y ** 3)
    return 1.13 * off + np.abs(oi.gelu_tanh(y)) * U * (8 + 4 * z)


SHAPES = [(1, 1, 1), (1, 16, 5), (3, 15, 33), (31, 17, 64), (33, 129, 65), (130, 127, 70), (257, 256, 136), (300, 1000, 129),
          (96, 384, 1152), (64, 4608, 40), (65, 64, 200), (129, 130, 257), (40, 385, 8)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_products(orch_lib, form, dtype, M, K, N):
    lib = orch_lib
    rng = np.random.default_rng(M * K + N)
    A, W, bias, s, *_ = _operands(lib, rng, M, K, N, gap=32 if M % 2 else 0)
    bd = to_dev(bias)
    for epi, b in ((lib.EPI_STORE, bd), (lib.EPI_STORE, None), (lib.EPI_GELU, bd)):
        out = torch.full((M + 1, N), 3.0, dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device=DEV)
        lib.linear_quantized(A, W, b, epi, out[:M])
        y = s + (0 if b is None else bias)
        # the sum to fp32, its two factors, the bias: four roundings
        off = 3 * U * np.abs(s) + U * np.abs(y)
        if epi == lib.EPI_GELU:
            _check(to_host(out)[:M], oi.gelu_tanh(y), _gelu_off(y, off), dtype)
        else:
            _check(to_host(out)[:M], y, off, dtype)
        assert torch.all(out[M] == 3.0)


@pytest.mark.parametrize("M,K,N,rpb", [(1, 20, 8, 1), (70, 200, 132, 1), (100, 144, 65, 33), (260, 128, 260, 260), (33, 1152, 31, 7)])
def test_gated_residual(orch_lib, form, M, K, N, rpb):
    lib = orch_lib
    rng = np.random.default_rng(M)
    A, W, bias, s, *_ = _operands(lib, rng, M, K, N)
    B = -(-M // rpb)
    for stride in (N, N + 4, N + 3):
        gate, h = rng.standard_normal((B, stride)).astype(np.float32), rng.standard_normal((M, N)).astype(np.float32)
        out = to_dev(h)
        lib.linear_quantized(A, W, to_dev(bias), lib.EPI_RESIDUAL, out, gate=to_dev(gate)[:, :N], rows_per_batch=rpb)
        y, g = s + bias, gate[np.arange(M) // rpb, :N].astype(np.float64)
        want = h + g * y
        _check(to_host(out), want, np.abs(g) * (3 * U * np.abs(s) + U * np.abs(y)), "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,n,K,heads,d,tokens,off", [
    (1, 1, 16, 1, 32, 1, 0), (2, 45, 200, 2, 72, 100, 13), (3, 33, 128, 3, 64, 64, 31), (2, 130, 144, 1, 128, 131, 1),
    (1, 96, 384, 6, 64, 256, 80), (2, 24, 96, 2, 80, 40, 16), (5, 7, 130, 1, 96, 9, 2)])
def test_qkv(orch_lib, form, dtype, B, n, K, heads, d, tokens, off):
    lib = orch_lib
    rng = np.random.default_rng(n)
    H = heads * d
    A, W, bias, s, *_ = _operands(lib, rng, B * n, K, 3 * H)
    y = s + bias
    for gap in (0, 16):
        kv = np.full((B, 2 * tokens * H + gap), 0.25)
        dt = torch.float32 if dtype == "f32" else torch.bfloat16
        q, kd = torch.empty((B, heads, n, d), dtype=dt, device=DEV), to_dev(kv, dtype)
        lib.qkv_projection_quantized(A, W, to_dev(bias), q, kd[:, :2 * tokens * H], tokens, off)
        wq, wkv = oi.qkv(y, B, heads, kv, tokens, off)
        eq, ekv = oi.qkv(3 * U * np.abs(s) + U * np.abs(y), B, heads, np.zeros_like(kv), tokens, off)
        _check(to_host(q), wq, eq, dtype)
        _check(to_host(kd), wkv, ekv, dtype)        # (tokens outside the band and behind a branch as they were)


def test_every_form_gives_the_same_bits(orch_lib, monkeypatch):
    """Sums are exact: neither the form nor M changes an output."""
    lib = orch_lib
    rng = np.random.default_rng(9)
    M, K, N = 300, 1111, 264
    A, W, bias, *_ = _operands(lib, rng, M, K, N)
    outs = []
    for f in FORMS:
        monkeypatch.setenv("ORCH_INT8_TILE", str(f))
        outs.append(torch.empty((M, N), dtype=torch.bfloat16, device=DEV))
        lib.linear_quantized(A, W, to_dev(bias), lib.EPI_STORE, outs[-1])
    monkeypatch.delenv("ORCH_INT8_TILE")
    values, scales = A.tensors
    one = torch.empty((1, N), dtype=torch.bfloat16, device=DEV)
    lib.linear_quantized(lib.int8_rows(values[77:78], scales[77:78]), W, to_dev(bias), lib.EPI_STORE, one)
    for o in outs:
        assert torch.equal(o, outs[0])
    assert torch.equal(one[0], outs[0][77])


def test_largest_sums(orch_lib, form):
    """131071 products of -128 and -128: the last sum that 32 bits hold."""
    lib = orch_lib
    K = 131071
    v = torch.full((2, 131072), -128, dtype=torch.int8, device=DEV)[:, :K]
    A = lib.int8_rows(v, torch.ones(2, device=DEV))
    out = torch.empty((2, 2), device=DEV)
    lib.linear_quantized(A, A, None, lib.EPI_STORE, out)
    assert torch.equal(out.cpu(), torch.full((2, 2), float(np.float32(16384.0 * K))))


def test_nan_rows_stay_in_their_rows(orch_lib, form):
    lib = orch_lib
    rng = np.random.default_rng(2)
    A, W, bias, s, *_ = _operands(lib, rng, 70, 100, 90)
    A.tensors[1][33] = float("nan")
    W.tensors[1][5] = float("nan")
    out = torch.empty((70, 90), device=DEV)
    lib.linear_quantized(A, W, to_dev(bias), lib.EPI_GELU, out)
    bad = torch.isnan(out).cpu()
    assert bad[33].all() and bad[:, 5].all() and int(bad.sum()) == 90 + 70 - 1


@pytest.mark.parametrize("shape", [(0, 64, 32), (0, 1, 1)])
def test_no_rows(orch_lib, shape):
    lib = orch_lib
    M, K, N = shape
    A = lib.int8_rows(torch.empty((0, 64), dtype=torch.int8, device=DEV)[:, :K], torch.empty(0, device=DEV))
    W = lib.int8_rows(torch.zeros((N, 64), dtype=torch.int8, device=DEV)[:, :K], torch.ones(N, device=DEV))
    lib.linear_quantized(A, W, None, lib.EPI_STORE, torch.empty((0, N), device=DEV))
    lib.quantize_rows(torch.empty((0, K), device=DEV), A)


@pytest.mark.parametrize("M,K,N", [(1, 12161, 24), (33, 13000, 72), (70, 16385, 96), (32, 131071, 40)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_split_k(orch_lib, dtype, M, K, N):
    """A long K over more workgroups: the same bits as without workspace, for every epilogue."""
    lib = orch_lib
    rng = np.random.default_rng(K)
    need = lib.linear_quantized_workspace_bytes(M, N, K)
    assert need > 0
    ws = torch.full((need // 4 + 4,), -7, dtype=torch.int32, device=DEV)
    A, W, bias, s, *_ = _operands(lib, rng, M, K, N, gap=16)
    bd, gate, dt = to_dev(bias), to_dev(rng.standard_normal((M, N))), torch.float32 if dtype == "f32" else torch.bfloat16
    h = to_dev(rng.standard_normal((M, N)))
    for epi in (lib.EPI_STORE, lib.EPI_GELU, lib.EPI_RESIDUAL):
        outs = []
        for w in (None, ws[:need // 4 - 1], ws[:need // 4]):
            outs.append(h.clone() if epi == lib.EPI_RESIDUAL else torch.empty((M, N), dtype=dt, device=DEV))
            lib.linear_quantized(A, W, bd, epi, outs[-1], gate=gate, rows_per_batch=1, workspace=w)
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
        if epi == lib.EPI_STORE:
            _check(to_host(outs[2]), s + bias, 3 * U * np.abs(s) + U * np.abs(s + bias), dtype)
    assert torch.all(ws[need // 4:] == -7)
    B, H = 1 if M % 2 else 2, 32 * 3
    if N == H:
        qk = []
        for w in (None, ws):
            q, kv = torch.empty((B, 1, M // B, 32), dtype=dt, device=DEV), torch.zeros((B, 2 * (M // B + 3) * 32), dtype=dt, device=DEV)
            lib.qkv_projection_quantized(A, W, bd, q, kv, M // B + 3, 2, workspace=w)
            qk.append((q, kv))
        assert torch.equal(qk[0][0], qk[1][0]) and torch.equal(qk[0][1], qk[1][1])


def test_far_rows(orch_lib, form):
    """Rows as far apart as they may be: the last of a tile 2^31 bytes behind its first."""
    lib = orch_lib
    rng = np.random.default_rng(11)
    M, K, N, far = 257, 200, 256, (1 << 23) - 16
    a, w = (rng.integers(-128, 128, (n, K), dtype=np.int8) for n in (M, N))
    buf = torch.empty((2 * M, far), dtype=torch.int8, device=DEV)       # A's rows, then W's
    ad, wd = buf[:M, :K], buf[M:M + N, 64:64 + K]
    ad.copy_(torch.from_numpy(a))
    wd.copy_(torch.from_numpy(w))
    one = torch.ones(M, device=DEV)
    out = torch.empty((M, N), device=DEV)
    lib.linear_quantized(lib.int8_rows(ad, one), lib.int8_rows(wd, one[:N]), None, lib.EPI_STORE, out)
    np.testing.assert_array_equal(to_host(out), oi.product(a, np.ones(M), w, np.ones(N)))


def test_wide_gates(orch_lib, form):
    """A gate for every token, as slices of a wider buffer."""
    lib = orch_lib
    rng = np.random.default_rng(12)
    M, K, N = 131, 64, 136
    A, W, bias, s, *_ = _operands(lib, rng, M, K, N)
    wide, h = rng.standard_normal((M, 6 * N)).astype(np.float32), rng.standard_normal((M, N)).astype(np.float32)
    gd, out = to_dev(wide), to_dev(h)
    lib.linear_quantized(A, W, to_dev(bias), lib.EPI_RESIDUAL, out, gate=gd[:, 2 * N:3 * N], rows_per_batch=1)
    g, y = wide[:, 2 * N:3 * N].astype(np.float64), s + bias
    _check(to_host(out), h + g * y, np.abs(g) * (3 * U * np.abs(s) + U * np.abs(y)), "f32")
