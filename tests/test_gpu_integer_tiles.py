"""8-bit integer products of many tiles: more than the persistent workgroups of the large tiles, several
groups of tile rows with a ragged last one, several k-tiles with a ragged last one.  Sums are exact and each
output is rounded by the same operations in every form, so all of a form's bits are compared with
those of 32 x 32 tiles (another kernel, whose outputs leave straight from the registers), and rows on both
sides of tiles' edges with the oracle."""
import numpy as np
import pytest
import torch

from oracle import integer as oi
from tests._gpu_util import DEV, to_dev, to_host

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": U, "bf16": 2.0 ** -8}
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
FORMS = range(6)
# 19 rows of 256 x 256 tiles (17 a row: 323), 25 of 192 x 256 (425), 37 of 128 x 128 (33 a row), 74 of 64 x 64 (66)
M, N = 4700, 4200
ROWS = [0, 63, 64, 127, 191, 192, 255, 256, 1023, 1024, 4095, 4096, 4607, 4608, 4671, 4672, M - 1]


def _operands(lib, M, K, N, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    held = lambda n: torch.randint(-128, 128, (n, -(-K // 16) * 16), dtype=torch.int8, device=DEV, generator=g)[:, :K]
    scales = lambda n: torch.exp(torch.randn(n, device=DEV, generator=g)) / (100 * K ** 0.5)
    A, W = lib.int8_rows(held(M), scales(M)), lib.int8_rows(held(N), scales(N))
    return A, W, torch.randn(N, device=DEV, generator=g)


def _host(r, rows=slice(None)):
    v, s = r.tensors
    return v[rows].cpu().numpy(), s[rows].cpu().numpy()


def _want(A, W, bias, rows):
    """Some rows in 64 bits, and what fp32 may be off: the sum, its two factors and the bias round once each."""
    s = oi.product(*_host(A, rows), *_host(W))
    y = s + (0 if bias is None else bias.cpu().numpy().astype(np.float64))
    return y, 3 * U * np.abs(s) + U * np.abs(y)


def _check(got, want, off, dtype):
    over = np.abs(got - want) - (HALF[dtype] * np.abs(want) + off * (1 + HALF[dtype]))
    assert (over <= 0).all(), (float(over.max()), np.unravel_index(over.argmax(), over.shape))


def _gelu(y, off):
    """GELU and its bound: y off by `off` moves it by 1.13 of that at most; its exponent is off by four roundings of
    itself, exp2 and the sum by three, the reciprocal and product by four (2^-22)."""
    z = 2 * np.sqrt(2 / np.pi) * np.abs(y + 0.044715 * y ** 3)
    w = oi.gelu_tanh(y)
    return w, 1.13 * off + np.abs(w) * U * (8 + 4 * z)


@pytest.fixture
def forms(monkeypatch):
    def run(call):
        """call() in 32 x 32 tiles, then (form, call()) of each other one."""
        monkeypatch.setenv("ORCH_INT8_TILE", "6")
        want = call()
        rest = []
        for f in FORMS:
            monkeypatch.setenv("ORCH_INT8_TILE", str(f))
            rest.append((f, call()))
        monkeypatch.delenv("ORCH_INT8_TILE")
        rest.append(("own", call()))
        torch.cuda.synchronize()
        return want, rest
    return run


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [100, 300])
@pytest.mark.parametrize("cols", [N, N + 1])            # whole 16-byte accesses, and an element each
@pytest.mark.parametrize("epilogue,with_bias", [("store", True), ("store", False), ("gelu", True)])
def test_every_bit(orch_lib, forms, dtype, K, cols, epilogue, with_bias):
    lib = orch_lib
    A, W, bias = _operands(lib, M, K, cols, K + cols)
    bias = bias if with_bias else None
    epi = lib.EPI_GELU if epilogue == "gelu" else lib.EPI_STORE

    def call():
        out = torch.full((M + 1, cols), 3.0, dtype=TYPE[dtype], device=DEV)
        lib.linear_quantized(A, W, bias, epi, out[:M])
        return out
    want, rest = forms(call)
    assert torch.all(want[M] == 3.0)
    y, off = _want(A, W, bias, ROWS)
    if epilogue == "gelu":
        y, off = _gelu(y, off)
    _check(to_host(want[ROWS]), y, off, dtype)
    for f, got in rest:
        assert torch.equal(got, want), f


@pytest.mark.parametrize("cols,rpb", [(N, 1567), (N + 2, 1), (N + 1, M)])
def test_every_bit_of_a_residual(orch_lib, forms, cols, rpb):
    """(the two large tiles have no such form: what the call picks by itself stands in for them)"""
    lib = orch_lib
    A, W, bias = _operands(lib, M, 300, cols, cols)
    B = -(-M // rpb)
    rng = np.random.default_rng(rpb)
    gate, h = to_dev(rng.standard_normal((B, cols))), to_dev(rng.standard_normal((M, cols)))

    def call():
        out = h.clone()
        lib.linear_quantized(A, W, bias, lib.EPI_RESIDUAL, out, gate=gate, rows_per_batch=rpb)
        return out
    want, rest = forms(call)
    y, off = _want(A, W, bias, ROWS)
    g = to_host(gate)[np.array(ROWS) // rpb]
    _check(to_host(want[ROWS]), to_host(h[ROWS]) + g * y, np.abs(g) * off, "f32")
    for f, got in rest:
        assert torch.equal(got, want), f


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,d,tokens,at", [(19, 72, 2400, 13), (20, 64, 2352, 0), (44, 32, 2355, 4)])
@pytest.mark.parametrize("K", [100, 300])
def test_every_bit_of_qkv(orch_lib, forms, dtype, heads, d, tokens, at, K):
    """Q, K and V^T of two branches; the column where V^T begins lies inside a tile (2736) or at an edge of
    every form's tiles (2560, 2816), and tiles of all three follow each other in a workgroup."""
    lib = orch_lib
    B, n, H = 2, 2350, heads * d
    A, W, bias = _operands(lib, B * n, K, 3 * H, heads + K)
    gap = 16

    def call():
        q = torch.empty((B, heads, n, d), dtype=TYPE[dtype], device=DEV)
        kv = torch.full((B, 2 * tokens * H + gap), 0.25, dtype=TYPE[dtype], device=DEV)
        lib.qkv_projection_quantized(A, W, bias, q, kv[:, :2 * tokens * H], tokens, at)
        return q, kv
    want, rest = forms(call)
    q, kv = want
    k, v = kv[:, :tokens * H].view(B, heads, tokens, d), kv[:, tokens * H:2 * tokens * H].view(B, heads, d, tokens)
    t = [0, 1, 7, 63, 255, 256, 1023, 2047, 2341, n - 1]
    for b in range(B):
        y, off = _want(A, W, bias, [b * n + i for i in t])
        parts = lambda x: x.reshape(len(t), 3, heads, d).transpose(1, 2, 0, 3)          # [3][heads][t][d]
        band = [at + i for i in t]
        got = torch.stack((q[b][:, t], k[b][:, band], v[b][:, :, band].transpose(1, 2)))
        _check(to_host(got), parts(y), parts(off), dtype)
    out = [i for i in range(tokens) if not at <= i < at + n]
    assert torch.all(k[:, :, out] == 0.25) and torch.all(v[..., out] == 0.25) and torch.all(kv[:, 2 * tokens * H:] == 0.25)
    for f, got in rest:
        assert torch.equal(got[0], q) and torch.equal(got[1], kv), f
