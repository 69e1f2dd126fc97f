"""The pass between two blocks against the oracle."""
import numpy as np
import pytest
import torch

from oracle import integer as oi
from tests._gpu_util import DEV, code, rounded, to_dev, to_host

pytestmark = pytest.mark.gpu

U = 2.0 ** -24                              # half a step of fp32
HALF = {"f32": U, "bf16": 2.0 ** -8}        # of the output's type


def _norm_error(x, kind, eps, e):
    """How far a row's norm (before its weight) may be off in fp32, x being off by e (both [rows, 1]-shaped
    bounds): the mean sums at most 36 channels a lane and 10 partial sums, so x - mean is off by 48 roundings of
    the row's largest magnitude; the sum of squares likewise by 48 of itself, its root by 24, root,
    reciprocal and product by 6 more; an error e of x moves the norm by 2 e / s."""
    top = np.abs(x).max(1, keepdims=True)
    if kind == "none":
        return e
    s = np.sqrt((x.var(1, keepdims=True) if kind == "layer" else (x * x).mean(1, keepdims=True)) + eps)
    return 2 * e / s + U * (48 * top / s + 32 * 2 * top / s)


def _bounds(h, y, post, pre, gate, shift, scale, rpb, a):
    """(h', u) in 64 bits, and how far fp32 may be off, per row."""
    n = h.shape[0]
    top = lambda v: np.abs(v).max(1, keepdims=True)
    h1, u = oi.block_norms(h, y, post, pre, gate, shift, scale, rpb, a)
    e = 2 * U * abs(a) * top(h) + 2 * U * top(h1)
    if y is not None:
        w = 1.0 if post[2] is None else np.abs(post[2]).max()
        g = 1.0 if gate is None else top(oi.rows_of(gate, n, rpb, None))
        z = oi.norm(y, *post)
        e = e + g * (w * _norm_error(y, post[0], post[1], 0.0) + 4 * U * top(z))
    w = 1.0 if pre[2] is None else np.abs(pre[2]).max()
    s = 1.0 if scale is None else top(1.0 + oi.rows_of(scale, n, rpb, None))
    v = oi.norm(h1, *pre)
    eu = s * (w * _norm_error(h1, pre[0], pre[1], e) + 4 * U * top(v)) + 4 * U * top(u)
    return h1, u, e, eu


def _check(got, want, e, dtype="f32"):
    assert got.shape == want.shape
    over = np.abs(got - want) - (HALF[dtype] * np.abs(want) + e * (1 + HALF[dtype]))
    assert (over <= 0).all(), (float(over.max()), np.unravel_index(over.argmax(), over.shape))


def _mod(rng, B, H):
    """gate, shift, scale in one buffer, as the conditioning leaves them."""
    return 0.3 * rng.standard_normal((B, 3, H)).astype(np.float32)


def _run(lib, rng, rows, H, dtype, post="rms", pre="layer", affine=True, mod=True, rpb=None, a=1.0, pads=(0, 0, 0, 0),
         y=True, want_h=True, want_u=True, in_place=False, codes=False, h=None, yv=None):
    rpb = rpb or max(1, rows // 2)
    B = -(-rows // rpb)
    hp, yp, hop, op = pads
    if h is None:
        h = (rng.standard_normal((rows, H)) * np.exp(rng.standard_normal((rows, 1))) + 3 * rng.standard_normal((1, H)))
    h = h.astype(np.float32).astype(np.float64)
    if yv is None:
        yv = rounded(rng.standard_normal((rows, H)) * np.exp(rng.standard_normal((1, H))), dtype)
    wb = [rng.standard_normal(H).astype(np.float32) if affine else None for _ in range(4)]
    m = _mod(rng, B, H)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    wide = lambda v, p, t: torch.cat((torch.full((rows, p), 9.0, dtype=t, device=DEV), v), 1)[:, p:]
    hd = wide(to_dev(h), hp, torch.float32)
    yd = wide(to_dev(yv, dtype), yp, dt) if y else None
    md = to_dev(m)
    g, t, s = (md[:, 0], md[:, 1], md[:, 2]) if mod else (None, None, None)
    dev = [None if w is None else to_dev(w) for w in wb]
    ho = hd if in_place else torch.full((rows, H + hop), 7.0, device=DEV)[:, hop:] if want_h else None
    out = out8 = None
    if want_u and codes:
        C = -(-H // 16) * 16 + 16
        out8 = lib.int8_rows(torch.full((rows, C), 77, dtype=torch.int8, device=DEV)[:, :H], torch.zeros(rows, device=DEV))
    elif want_u:
        out = yd if in_place and y else torch.full((rows, H + op), 5.0, dtype=dt, device=DEV)[:, op:]
    lib.block_norms(hd, yd, ho, out8 if codes else out, post=lib.norm(post, 1e-6, dev[0], dev[1]),
                    pre=lib.norm(pre, 1e-5, dev[2], dev[3]), gate=g, shift=t, scale=s, rows_per_batch=rpb, residual_scale=a)
    none = (None, None, None)
    ms = (m[:, 0], m[:, 1], m[:, 2]) if mod else none
    h1, u, e, eu = _bounds(h, yv if y else None, (post, 1e-6, wb[0], wb[1]), (pre, 1e-5, wb[2], wb[3]), *ms, rpb, a)
    if want_h:
        _check(to_host(ho), h1, e)
        if hop:
            assert torch.all(ho.as_strided((rows, hop), (H + hop, 1), 0) == 7.0)
    if want_u and codes:
        values, scales = out8.tensors
        sc = scales.cpu().numpy().astype(np.float64)[:, None]
        top = np.abs(u).max(1, keepdims=True)
        np.testing.assert_array_less(np.abs(sc * 127 - top), eu + 2 * U * top + 1e-300)
        # half a code, its two roundings at 127, what the row itself is off by, and its largest value's share of it
        _check(values.cpu().numpy() * sc, u, sc * (0.5 + 127 * 4 * U) + 2 * eu)
        assert np.abs(values.cpu().numpy()).max(1).min() == 127
        assert torch.all(values.as_strided((rows, 16), (values.stride(0), 1), -(-H // 16) * 16) == 77)
    elif want_u:
        _check(to_host(out), u, eu, dtype)


# widths: one lane's, odd ones, each kernel form's first and last, the widest
WIDTHS = [1, 3, 4, 31, 32, 100, 128, 384, 388, 511, 513, 1021, 1152, 1156, 2304, 2305, 2308, 9216, 9217, 9220]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H", WIDTHS)
@pytest.mark.parametrize("codes", [False, True])
def test_widths(orch_lib, dtype, H, codes):
    _run(orch_lib, np.random.default_rng(H), 5, H, dtype, codes=codes)


@pytest.mark.parametrize("H", [32768, 32767])
def test_widest(orch_lib, H):
    _run(orch_lib, np.random.default_rng(H), 3, H, "bf16")
    _run(orch_lib, np.random.default_rng(H), 3, H, "f32", codes=True)


@pytest.mark.parametrize("post", ["none", "layer", "rms"])
@pytest.mark.parametrize("pre", ["none", "layer", "rms"])
@pytest.mark.parametrize("affine,mod", [(False, False), (True, True), (False, True)])
def test_kinds(orch_lib, post, pre, affine, mod):
    for dtype, a in (("bf16", 1.0), ("f32", -0.5)):
        _run(orch_lib, np.random.default_rng(3), 37, 132, dtype, post, pre, affine, mod, rpb=11, a=a)


@pytest.mark.parametrize("rows,rpb", [(1, 1), (2, 1), (7, 7), (8, 3), (9, 100), (257, 64), (1025, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows(orch_lib, dtype, rows, rpb):
    _run(orch_lib, np.random.default_rng(rows), rows, 96, dtype, rpb=rpb)


@pytest.mark.parametrize("pads", [(4, 8, 4, 8), (1, 0, 0, 0), (0, 1, 0, 0), (0, 2, 0, 4), (0, 0, 3, 0), (0, 0, 0, 1), (5, 7, 9, 11)])
@pytest.mark.parametrize("H", [64, 61, 1152])
def test_strides(orch_lib, H, pads):
    for dtype in ("bf16", "f32"):
        _run(orch_lib, np.random.default_rng(H), 19, H, dtype, pads=pads)


@pytest.mark.parametrize("H", [45, 1152, 4608, 12000])
def test_in_place(orch_lib, H):
    for dtype in ("bf16", "f32"):
        _run(orch_lib, np.random.default_rng(H), 21, H, dtype, in_place=True)


@pytest.mark.parametrize("H", [45, 1152])
def test_parts(orch_lib, H):
    """The first block's (no block before it) and the last one's (none behind it)."""
    rng = np.random.default_rng(1)
    _run(orch_lib, rng, 9, H, "bf16", y=False)
    _run(orch_lib, rng, 9, H, "f32", y=False, want_h=False, a=2.0)
    _run(orch_lib, rng, 9, H, "bf16", want_u=False)
    _run(orch_lib, rng, 9, H, "bf16", want_h=False)
    _run(orch_lib, rng, 9, H, "bf16", want_h=False, codes=True)


def test_far_from_zero(orch_lib):
    """Channels 1000 deviations from zero: the variance about the mean keeps its places."""
    rng = np.random.default_rng(4)
    h = 1000.0 + rng.standard_normal((6, 1152))
    _run(orch_lib, rng, 6, 1152, "f32", h=h, yv=rounded(0.01 * rng.standard_normal((6, 1152)), "f32"), affine=False)


def test_constant_rows(orch_lib):
    """No variance: eps alone divides; a row of zeros has codes and scale 0."""
    lib = orch_lib
    h = torch.zeros((4, 64), device=DEV)
    h[1], h[2] = 5.0, -3.0
    out = torch.empty_like(h)
    lib.block_norms(h, None, None, out, pre=lib.norm("layer", 1e-6))
    assert torch.equal(out, torch.zeros_like(out))
    q = lib.int8_rows(torch.full((4, 64), 3, dtype=torch.int8, device=DEV), torch.full((4,), 3.0, device=DEV))
    lib.block_norms(h, None, None, q, pre=lib.norm("layer", 1e-6))
    assert not q.tensors[0].any() and not q.tensors[1].any()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("H", [60, 61, 1152, 2400, 12000])
def test_not_finite_stays_in_its_row(orch_lib, bad, H):
    lib = orch_lib
    rng = np.random.default_rng(5)
    h, y = rng.standard_normal((11, H)).astype(np.float32), rng.standard_normal((11, H)).astype(np.float32)
    runs = []
    for plant in (False, True):
        hd, yd = to_dev(h), to_dev(y)
        if plant:
            hd[3, H // 2], yd[7, H - 1] = bad, bad
        ho, out = torch.empty_like(hd), torch.empty_like(hd)
        q = lib.int8_rows(torch.zeros((11, -(-H // 16) * 16), dtype=torch.int8, device=DEV)[:, :H], torch.zeros(11, device=DEV))
        for o in (out, q):
            lib.block_norms(hd, yd, ho, o, post=lib.norm("rms"), pre=lib.norm("layer"))
        runs.append((ho, out, *q.tensors))
    rows = [r for r in range(11) if r not in (3, 7)]
    for a, b in zip(*runs):
        assert torch.equal(a[rows], b[rows])
    ho, out, values, scales = runs[1]
    assert torch.isnan(out[[3, 7]]).all()
    assert torch.isnan(scales[[3, 7]]).all() and not values[[3, 7]].any()


def test_no_rows(orch_lib):
    e = torch.empty((0, 64), device=DEV)
    orch_lib.block_norms(e, None, None, torch.empty((0, 64), device=DEV), pre=orch_lib.norm("layer"))


def test_replaces_the_layernorm(orch_lib):
    """Without a block before it the pass is orch_op_layernorm_modulate, to the last roundings."""
    lib = orch_lib
    rng = np.random.default_rng(6)
    h, m = to_dev(rng.standard_normal((200, 1152))), to_dev(_mod(rng, 2, 1152))
    a, b = (torch.empty((200, 1152), device=DEV) for _ in range(2))
    lib.layernorm_modulate(h, 200, 1152, 100, m[:, 1], m[:, 2], 3 * 1152, a, code("f32"))
    lib.block_norms(h, None, None, b, pre=lib.norm("layer", 1e-6), shift=m[:, 1], scale=m[:, 2], rows_per_batch=100)
    # both are off by 48 + 64 roundings of 8 deviations at most, times 1 + scale below 4
    assert float((a - b).abs().max()) < 2 * U * (48 + 64) * 8 * 4
