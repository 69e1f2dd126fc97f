"""Rotary positions against the float64 oracle.

Tolerance, elementwise: half a step of the output's type (bf16 2^-8, fp32 2^-24 of
the value) and what fp32 loses on the way, in units of |x| + |y| of the pair: the
turn's fraction rounded to fp32 (at most 2^-26 turns, 2^-23.3 radians), sine and cosine (2 ulp: 2^-23
each), two products and a sum (2^-24 each): under 2^-21 together.
"""
import numpy as np
import pytest
import torch

from oracle import kvcache as ok
from tests._gpu_util import DEV, rounded, to_dev, to_host

pytestmark = pytest.mark.gpu


def _check(got, x, ref, dtype):
    size = np.abs(x).max(-1, keepdims=True) * 2
    tol = np.abs(ref) * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) + size * 2.0 ** -21
    assert (np.abs(got - ref) <= tol).all(), float((np.abs(got - ref) / tol).max())


# channels, extent, token_begin, n_tok, origin, step, theta
GRIDS = {
    "one token": ((0, 16, 16), (1, 1, 1), 0, 1, (0, 0, 0), (1, 1, 1), 1e4),
    "band": ((0, 16, 16), (1, 12, 12), 36, 48, (0, -5.5, -5.5), (1, 1, 1), 1e4),
    "video": ((4, 12, 14), (5, 7, 9), 40, 211, (0, 0, 0), (1, 0.5, 0.5), 256.0),
    "some pass": ((2, 6, 10), (3, 5, 7), 1, 104, (0, 0, 0), (1, 1, 1), 100.0),
    "time only": ((32, 0, 0), (1000, 1, 1), 17, 500, (0, 0, 0), (1, 1, 1), 1e4),
    "none": ((0, 0, 0), (1, 8, 8), 0, 64, (0, 0, 0), (1, 1, 1), 1e4),
    "far": ((16, 8, 8), ((1 << 20) - 1, 32, 64), 2 ** 31 - 2048 - 301, 301, (1e6, 0, 0), (1, 1, 1), 1e4),
    "wide": ((0, 16, 16), (1, 40, 60), 0, 2400, (0, 4096, 4096), (1, 1, 1), 1e6),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("name", GRIDS)
@pytest.mark.parametrize("B,heads,d", [(1, 1, 32), (2, 3, 72), (1, 6, 64), (2, 2, 128)])
def test_rotary(orch_lib, dtype, interleaved, name, B, heads, d):
    ch, ext, begin, n, origin, step, theta = GRIDS[name]
    if name == "band" and d == 72:
        ch = (0, 36, 36)
    if name == "video" and d == 128:
        ch = (16, 56, 56)
    ax = orch_lib.rotary_axes(ch, ext, theta, origin, step, interleaved)
    rng = np.random.default_rng(d + n)
    x = rounded(rng.standard_normal((B, heads, n, d)) * 3, dtype)
    xd = to_dev(x, dtype)
    out = torch.full_like(xd, float("nan"))
    orch_lib.rotary(ax, begin, xd, out)
    ref = ok.rotary(x, begin, ch, ext, origin, step, theta, interleaved)
    _check(to_host(out), x, ref, dtype)
    # channels past the axes' are copies
    assert torch.equal(out[..., sum(ch):], xd[..., sum(ch):])
    # in place: the same bits
    orch_lib.rotary(ax, begin, xd, xd)
    assert torch.equal(xd, out)


@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_two_tensors_with_strides(orch_lib, dtype, interleaved):
    """Q and K out of a packed token-major projection (K with fewer heads), at an odd
    element offset, into a K buffer's band: one launch; the rest of both buffers untouched."""
    B, heads, kh, n, d = 2, 4, 2, 33, 64
    ch, ext = (0, 24, 32), (1, 9, 11)
    ax = orch_lib.rotary_axes(ch, ext, 1e4, interleaved=interleaved)
    rng = np.random.default_rng(5)
    W = (heads + kh) * d
    x = rounded(rng.standard_normal(1 + B * n * W), dtype)
    xd = to_dev(x, dtype)
    packed = xd[1:].view(B, n, heads + kh, d)
    q, k = packed[:, :, :heads].transpose(1, 2), packed[:, :, heads:].transpose(1, 2)
    qo = torch.full((B, heads, n, d), 7.0, dtype=xd.dtype, device=DEV)
    buf = torch.full((B, kh, 99, d), 7.0, dtype=xd.dtype, device=DEV)
    ko = buf[:, :, 22:22 + n]
    orch_lib.rotary(ax, 22, (q, k), (qo, ko))
    xr = x[1:].reshape(B, n, heads + kh, d).transpose(0, 2, 1, 3)
    ref = ok.rotary(xr, 22, ch, ext, (0, 0, 0), (1, 1, 1), 1e4, interleaved)
    _check(to_host(qo), xr[:, :heads], ref[:, :heads], dtype)
    _check(to_host(ko), xr[:, heads:], ref[:, heads:], dtype)
    assert torch.all(buf[:, :, :22] == 7.0) and torch.all(buf[:, :, 22 + n:] == 7.0)
    assert torch.equal(xd, to_dev(x, dtype))
    # in place, the other part of the packed buffer untouched
    orch_lib.rotary(ax, 22, k, k)
    assert torch.equal(k, ko) and torch.equal(q, to_dev(x, dtype)[1:].view(B, n, heads + kh, d)[:, :, :heads].transpose(1, 2))


def test_inverse_and_gradient(orch_lib):
    """Negated steps undo the rotation; the gradient of g . rotate(x) is the inverse rotation of g, by differences."""
    ch, ext, n, d = (4, 12, 16), (2, 5, 6), 60, 32
    fwd = orch_lib.rotary_axes(ch, ext, 1e4, (0.0, -2.0, 3.0))
    inv = orch_lib.rotary_axes(ch, ext, 1e4, (0.0, -2.0, 3.0), (-1.0, -1.0, -1.0))
    rng = np.random.default_rng(2)
    x, g = (rng.standard_normal((1, 2, n, d)).astype(np.float32) for _ in range(2))
    xd, y, back, grad = to_dev(x), torch.empty((1, 2, n, d), device=DEV), torch.empty((1, 2, n, d), device=DEV), torch.empty((1, 2, n, d), device=DEV)
    orch_lib.rotary(fwd, 0, xd, y)
    orch_lib.rotary(inv, 0, y, back)
    assert np.abs(to_host(back) - x).max() <= 2.0 ** -19 * np.abs(x).max()
    orch_lib.rotary(inv, 0, to_dev(g), grad)
    gr, h = to_host(grad), 1e-3
    for i in [(0, 0, 0, 0), (0, 1, 7, 5), (0, 0, 59, 31), (0, 1, 30, 17)]:
        a, b = x.astype(np.float64), x.astype(np.float64)
        a[i] += h
        b[i] -= h
        f = [(ok.rotary(v, 0, ch, ext, (0.0, -2.0, 3.0), (1, 1, 1), 1e4, True) * g).sum() for v in (a, b)]
        assert gr[i] == pytest.approx((f[0] - f[1]) / (2 * h), abs=1e-5)


def test_not_finite_stays_in_its_pair(orch_lib):
    ax = orch_lib.rotary_axes((0, 8, 8), (1, 4, 4))
    x = torch.randn((1, 2, 16, 32), device=DEV)
    x[0, 0, 5, 2] = float("nan")
    x[0, 1, 9, 20] = float("inf")
    out = torch.empty_like(x)
    orch_lib.rotary(ax, 0, x, out)
    bad = ~torch.isfinite(out)
    assert bad.nonzero().tolist() == [[0, 0, 5, 2], [0, 0, 5, 3], [0, 1, 9, 20]]


def test_no_tokens(orch_lib):
    ax = orch_lib.rotary_axes((0, 16, 16), (1, 4, 4))
    x = torch.ones((2, 3, 8, 32), device=DEV)
    ts = (orch_lib.RotaryTensor * 1)()
    ts[0].x = ts[0].out = x.data_ptr()
    ts[0].heads = 3
    orch_lib.check(orch_lib.lib.orch_op_rotary(orch_lib.C.byref(ax), ts, 1, 2, 0, 16, 32, 0, None))
    torch.cuda.synchronize()
    assert torch.all(x == 1)


@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("theta", [1.0001, 2.0, 100.0])
def test_far_origin(orch_lib, theta, interleaved):
    """Positions of 10^12, 64 pairs of one axis: every pair's angle is off by two fp64 roundings (the pair's turns per
    position, and their product with the position: 2^-52 of the angle) and what _check allows for, whatever its number.
    Angles of the reference in 80 bits, where those two roundings are 2^-63."""
    n, d, origin = 64, 128, 1e12
    ax = orch_lib.rotary_axes((d, 0, 0), (n, 1, 1), theta, (origin, 0, 0), (1, 1, 1), interleaved)
    x = np.random.default_rng(3).standard_normal((1, 2, n, d)).astype(np.float32)
    out = torch.empty((1, 2, n, d), device=DEV)
    orch_lib.rotary(ax, 0, to_dev(x), out)
    assert np.finfo(np.longdouble).nmant >= 63
    i = np.arange(d // 2).astype(np.longdouble)
    phi = (np.longdouble(origin) + np.arange(n))[:, None] * np.longdouble(theta) ** (-2 * i / d)
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :d // 2], x[..., d // 2:])
    u, v = np.cos(phi) * a - np.sin(phi) * b, np.sin(phi) * a + np.cos(phi) * b
    got = to_host(out)
    gu, gv = (got[..., 0::2], got[..., 1::2]) if interleaved else (got[..., :d // 2], got[..., d // 2:])
    tol = (np.abs(a) + np.abs(b)) * (2.0 ** -21 + 2.0 ** -52 * phi) + 2.0 ** -24 * (np.abs(u) + np.abs(v))
    for g, ref in ((gu, u), (gv, v)):
        print(float((np.abs(g - ref) / tol).max()), flush=True)
        assert (np.abs(g - ref) <= tol).all()


def test_in_place_whatever_the_stride_of_one(orch_lib):
    """The stride of an extent of one has no meaning: in place with another one there."""
    ax = orch_lib.rotary_axes((0, 16, 16), (1, 4, 4))
    x = torch.randn((1, 2, 1, 32), device=DEV)
    want = torch.empty_like(x)
    orch_lib.rotary(ax, 5, x, want)
    orch_lib.rotary(ax, 5, x, x.as_strided(x.shape, (999, 32, 7, 1)))
    assert torch.equal(x, want)
