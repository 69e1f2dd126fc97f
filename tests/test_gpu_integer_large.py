"""The norms around a block and the 8-bit integer products at sizes past 32 bits of one kind or another."""
import numpy as np
import pytest
import torch

from oracle import integer as oi
from tests._gpu_util import DEV, to_host

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def test_wide_rows_past_a_grid(orch_lib):
    """2^22 rows and more of a workgroup of 1024 threads each: more threads than 32 bits count.  In place,
    so that a row that is taken twice or not at all shows."""
    lib = orch_lib
    rows, H = (1 << 22) + 3, 5124                        # 86 GB
    free, _ = torch.cuda.mem_get_info()
    if free < 100 << 30:
        pytest.skip("needs 100 GiB of free device memory")
    h = torch.ones((rows, H), device=DEV)
    some = [0, 1, (1 << 21) - 1, 1 << 21, (1 << 21) + 1, (1 << 22) - 1, 1 << 22, rows - 1]
    x = np.random.default_rng(0).standard_normal((len(some), H)).astype(np.float32)
    for i, r in enumerate(some):
        h[r] = torch.from_numpy(x[i]).to(DEV)
    lib.block_norms(h, None, h, residual_scale=0.5)
    torch.cuda.synchronize()
    for i, r in enumerate(some):
        np.testing.assert_array_equal(h[r].cpu().numpy(), 0.5 * x[i])
        h[r] = 0.5
    for part in h.split(1 << 18):
        lo, hi = torch.aminmax(part)
        assert float(lo) == 0.5 and float(hi) == 0.5
    del h, part
    torch.cuda.empty_cache()


def _codes(M, N, K, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    a, w = (torch.randint(-127, 128, (n, K), dtype=torch.int8, device=DEV, generator=g) for n in (M, N))
    sa, sw = (torch.rand(n, device=DEV, generator=g) for n in (M, N))
    return a, sa, w, sw, torch.randn(N, device=DEV, generator=g)


def _want(a, sa, w, sw, bias, rows):
    """Outputs of some rows in 64 bits, and what fp32 may be off: the sum, its two factors and the bias round once each."""
    s = oi.product(a[rows].cpu().numpy(), sa[rows].cpu().numpy(), w.cpu().numpy(), sw.cpu().numpy())
    y = s + bias.cpu().numpy()
    return y, 3 * U * np.abs(s) + U * np.abs(y)


def _check(got, want, off, half):
    assert (np.abs(got - want) <= half * np.abs(want) + off * (1 + half)).all()


def test_residual_past_32_bits(orch_lib):
    """A residual stream of more than 2^31 elements, 8.7 GB."""
    lib = orch_lib
    M, K, N, rpb = 460000, 32, 4736, 230001
    a, sa, w, sw, bias = _codes(M, N, K, 1)
    gate = torch.randn((2, N), device=DEV)
    out = torch.full((M, N), 0.25, device=DEV)
    lib.linear_quantized(lib.int8_rows(a, sa), lib.int8_rows(w, sw), bias, lib.EPI_RESIDUAL, out, gate=gate, rows_per_batch=rpb)
    rows = torch.tensor([0, 1, rpb - 1, rpb, 453437, 453438, M - 257, M - 1], device=DEV)
    y, off = _want(a, sa, w, sw, bias, rows)
    g = gate.cpu().numpy().astype(np.float64)[rows.cpu().numpy() // rpb]
    _check(to_host(out[rows]), 0.25 + g * y, np.abs(g) * off, U)


def test_qkv_past_32_bits(orch_lib):
    """Q of more than 2^31 elements, a K/V buffer of two branches of as many each, 13 GB."""
    lib = orch_lib
    B, n, K, heads, d, tokens, off = 2, 230000, 32, 74, 64, 230011, 5
    H = heads * d
    a, sa, w, sw, bias = _codes(B * n, 3 * H, K, 2)
    q = torch.empty((B, heads, n, d), dtype=torch.bfloat16, device=DEV)
    kv = torch.full((B, 2 * tokens * H), 9.0, dtype=torch.bfloat16, device=DEV)
    lib.qkv_projection_quantized(lib.int8_rows(a, sa), lib.int8_rows(w, sw), bias, q, kv, tokens, off)
    k, v = kv[:, :tokens * H].view(B, heads, tokens, d), kv[:, tokens * H:].view(B, heads, d, tokens)
    t = torch.tensor([0, 1, 113355, 226720, n - 257, n - 1], device=DEV)
    for b in range(B):
        y, e = _want(a, sa, w, sw, bias, b * n + t)
        parts = lambda x: x.reshape(len(t), 3, heads, d).transpose(1, 2, 0, 3)          # [3][heads][t][d]
        got = torch.stack((q[b][:, t], k[b][:, off + t], v[b][:, :, off + t].transpose(1, 2)))
        _check(to_host(got), parts(y), parts(e), 2.0 ** -8)
    for i in (*range(off), *range(off + n, tokens)):                                    # around the band
        assert bool((k[:, :, i] == 9.0).all()) and bool((v[..., i] == 9.0).all())
