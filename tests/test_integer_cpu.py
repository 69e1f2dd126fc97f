"""CPU side of the norms around a block, the quantiser of rows and the 8-bit integer
products: the oracle's pins, and every call that the library refuses (checked
before anything is launched, so no GPU is needed; the pointers are never read)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import integer as oi

F32, BF16 = 0, 1
P = [0x10000000 * (i + 1) for i in range(16)]      # addresses far apart, 16-byte aligned


# ---- the oracle ------------------------------------------------------------------

def test_norms_are_torchs():
    rng = np.random.default_rng(0)
    x, w, b = rng.standard_normal((5, 40)) + 2.0, rng.standard_normal(40), rng.standard_normal(40)
    t = torch.from_numpy(x)
    want = torch.nn.functional.layer_norm(t, (40,), torch.from_numpy(w), torch.from_numpy(b), 1e-5).numpy()
    np.testing.assert_allclose(oi.norm(x, "layer", 1e-5, w, b), want, rtol=1e-12, atol=1e-12)
    want = torch.nn.functional.rms_norm(t, (40,), torch.from_numpy(w), 1e-5).numpy()
    np.testing.assert_allclose(oi.norm(x, "rms", 1e-5, w), want, rtol=1e-12, atol=1e-12)


def test_block_norms_by_hand():
    h, y = np.array([[1.0, 3.0], [2.0, -2.0]]), np.array([[3.0, 4.0], [0.0, 2.0]])
    gate, shift, scale = np.array([[2.0, 0.5]]), np.array([[0.0, 1.0]]), np.array([[1.0, 0.0]])
    h1, u = oi.block_norms(h, y, ("rms", 0.0), ("layer", 0.0), gate, shift, scale, 2, 0.5)
    r = np.sqrt(12.5)
    np.testing.assert_allclose(h1, [[0.5 + 6 / r, 1.5 + 2 / r], [1.0, -1.0 + 1 / np.sqrt(2)]], rtol=1e-15)
    s = np.sign(h1[:, :1] - h1[:, 1:])                                   # two channels: +-1 after a LayerNorm
    np.testing.assert_allclose(u, np.concatenate([2 * s, 1 - s], 1), rtol=1e-12)


def test_codes_are_the_nearest():
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((200, 9)) * 2.0 ** rng.integers(-100, 100, (200, 1))).astype(np.float32)
    q, s = oi.quantize_rows(x)
    assert np.abs(q).max(1).min() == 127
    # half a code, and the two roundings of its quotient
    assert (np.abs(q * s[:, None].astype(np.float64) - x) <= s[:, None] * (0.5 + 127 * 4 * 2.0 ** -24)).all()


def test_ties_go_to_even_and_special_rows():
    x = np.array([[127, 0.5, 1.5, -2.5, -0.5], [0, 0, 0, 0, 0], [1, np.inf, 0, 0, 0], [np.nan, 1, 0, 0, 0],
                  [2.0 ** -149, 0, 0, 0, -2.0 ** -149]], np.float32)
    q, s = oi.quantize_rows(x)
    np.testing.assert_array_equal(q, [[127, 0, 2, -2, 0], [0] * 5, [0] * 5, [0] * 5, [127, 0, 0, 0, -127]])
    assert s[0] == 1 and s[1] == 0 and np.isnan(s[2]) and np.isnan(s[3]) and s[4] == 0


def test_product_is_the_loop():
    rng = np.random.default_rng(2)
    a, w = rng.integers(-128, 128, (3, 7), dtype=np.int8), rng.integers(-128, 128, (4, 7), dtype=np.int8)
    y = oi.product(a, [1, 2, 0.5], w, [1, 3, 1, 2], [0, 0, 1, 0])
    for m in range(3):
        for n in range(4):
            s = sum(int(a[m, k]) * int(w[n, k]) for k in range(7))
            assert y[m, n] == s * [1, 2, 0.5][m] * [1, 3, 1, 2][n] + [0, 0, 1, 0][n]


def test_qkv_places():
    y = np.arange(2 * 3 * 12, dtype=np.float64).reshape(6, 12)            # B 2, 3 tokens, 2 heads of 2
    q, kv = oi.qkv(y, 2, 2, np.zeros((2, 2 * 5 * 4)), 5, 1)
    assert q[1, 1, 2, 0] == y[5, 2]
    assert kv[1, (1 * 5 + 1 + 2) * 2 + 1] == y[5, 4 + 3]                   # K head 1, token 3, channel 1
    assert kv[1, 20 + (1 * 2 + 1) * 5 + 1 + 2] == y[5, 8 + 3]              # V^T head 1, channel 1, token 3


# ---- refusals --------------------------------------------------------------------

def _refused(lib, rc, word):
    assert rc == lib.ORCH_EINVAL
    assert word in lib.last_error(), lib.last_error()


def _i8(lib, values, scales, stride):
    return lib.Int8Rows(values, scales, stride)


def _norms(lib, dtype=BF16, out8=None, **kw):
    p = lib.BlockNorms()
    d = dict(rows=6, hidden=32, rows_per_batch=3, residual_scale=1.0, h=P[0], y=P[1], gate=P[2], shift=P[3], scale=P[4],
             h_out=P[5], out=P[6], h_stride=32, y_stride=32, mod_stride=32, h_out_stride=32, out_stride=32)
    d.update({k: v for k, v in kw.items() if "_" not in k or k in d})
    for k, v in d.items():
        setattr(p, k, v)
    for n in ("post", "pre"):
        m = getattr(p, n)
        m.kind, m.eps = kw.get(n + "_kind", 1), kw.get(n + "_eps", 1e-6)
        m.weight, m.bias = kw.get(n + "_weight"), kw.get(n + "_bias")
    if out8 is not None:
        p.out8 = C.pointer(_i8(lib, *out8))
    return lib.lib.orch_op_block_norms(C.byref(p), dtype, None)


INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("kw,word", [
    (dict(dtype=2), "dtype"), (dict(rows=-1), "shape"), (dict(rows=1 << 24), "shape"), (dict(hidden=0), "shape"),
    (dict(hidden=32769), "shape"), (dict(residual_scale=NAN), "residual_scale"), (dict(residual_scale=INF), "residual_scale"),
    (dict(post_kind=3), "post"), (dict(pre_kind=-1), "pre"), (dict(post_eps=0.0), "eps"), (dict(pre_eps=-1.0), "eps"),
    (dict(pre_eps=NAN), "eps"), (dict(post_eps=INF), "eps"), (dict(h=None), "NULL"),
    (dict(h_out=None, out=None), "nothing to write"), (dict(out8=(P[7], P[8], 32)), "exclude"),
    (dict(rows_per_batch=0), "rows_per_batch"), (dict(rows_per_batch=-3), "rows_per_batch"), (dict(mod_stride=31), "mod_stride"),
    (dict(mod_stride=1 << 40), "mod_stride"), (dict(h_stride=31), "strides"), (dict(y_stride=0), "strides"),
    (dict(h_out_stride=16), "strides"), (dict(out_stride=1 << 40), "strides"), (dict(h=P[0] + 2), "aligned"),
    (dict(y=P[1] + 1), "aligned"), (dict(y=P[1] + 2, dtype=F32), "aligned"), (dict(gate=P[2] + 1), "aligned"),
    (dict(shift=P[3] + 2), "aligned"), (dict(scale=P[4] + 3), "aligned"), (dict(h_out=P[5] + 1), "aligned"),
    (dict(out=P[6] + 1), "aligned"), (dict(post_weight=P[9] + 2), "aligned"), (dict(pre_bias=P[9] + 1), "aligned"),
    (dict(out=None, out8=(None, P[8], 32)), "NULL"), (dict(out=None, out8=(P[7], None, 32)), "NULL"),
    (dict(out=None, out8=(P[7] + 8, P[8], 32)), "16-byte"), (dict(out=None, out8=(P[7], P[8] + 2, 32)), "aligned"),
    (dict(out=None, out8=(P[7], P[8], 40)), "multiple of 16"), (dict(out=None, out8=(P[7], P[8], 16)), "multiple of 16"),
    (dict(out=None, out8=(P[7], P[8], 1 << 23)), "2^23"),
    (dict(h_out=P[0] + 64), "overlaps"), (dict(h_out=P[0], h_out_stride=64), "overlaps"), (dict(out=P[0]), "overlaps"),
    (dict(out=P[1] + 2), "overlaps"), (dict(out=P[1], out_stride=40), "overlaps"), (dict(h_out=P[2]), "overlaps"),
    (dict(out=P[3] + 4), "overlaps"), (dict(h_out=P[9], pre_weight=P[9]), "overlaps"), (dict(out=P[5]), "overlap"),
    (dict(out=None, out8=(P[5], P[8], 32)), "overlap"), (dict(out=None, out8=(P[7], P[7] + 16, 32)), "overlap"),
    (dict(out=None, out8=(P[1], P[8], 64)), "overlap"),
])
def test_block_norms_refuses(orch_lib, kw, word):
    _refused(orch_lib, _norms(orch_lib, **kw), word)


def test_block_norms_null_struct(orch_lib):
    _refused(orch_lib, orch_lib.lib.orch_op_block_norms(None, BF16, None), "NULL")


def test_no_rows_need_no_buffers(orch_lib):
    lib = orch_lib
    assert _norms(lib, rows=0, h=None, y=None, gate=None, shift=None, scale=None, h_out=None, out=None) == 0
    assert lib.lib.orch_op_quantize_rows(None, 0, 0, 8, None, BF16, None) == 0
    assert lib.lib.orch_op_linear_quantized(None, 0, 8, None, 8, None, 0, None, 0, 0, None, None, 0, BF16, None) == 0
    assert lib.lib.orch_op_qkv_projection_quantized(None, 2, 0, 8, None, None, 2, 32, None, None, 0, 4, 0, None, 0, BF16, None) == 0


def _quantize(lib, x=P[0], xs=40, rows=5, cols=40, out=(P[1], P[2], 48), dtype=BF16):
    o = None if out is None else C.byref(_i8(lib, *out))
    return lib.lib.orch_op_quantize_rows(x, xs, rows, cols, o, dtype, None)


@pytest.mark.parametrize("kw,word", [
    (dict(dtype=7), "dtype"), (dict(rows=-1), "shape"), (dict(rows=1 << 24), "shape"), (dict(cols=0), "shape"),
    (dict(cols=131072), "shape"), (dict(x=None), "NULL"), (dict(xs=39), "x_stride"), (dict(xs=1 << 40), "x_stride"),
    (dict(x=P[0] + 1), "aligned"), (dict(x=P[0] + 2, dtype=F32), "aligned"), (dict(out=None), "NULL"),
    (dict(out=(P[1], P[2], 47)), "multiple of 16"), (dict(out=(P[1], P[2], 32)), "multiple of 16"),
    (dict(out=(P[1] + 4, P[2], 48)), "16-byte"), (dict(out=(P[0] + 16, P[2], 48)), "overlap"),
    (dict(out=(P[1], P[0] + 4, 48)), "overlap"), (dict(out=(P[1], P[1] + 48, 48)), "overlap"),
])
def test_quantize_refuses(orch_lib, kw, word):
    _refused(orch_lib, _quantize(orch_lib, **kw), word)


def _linear(lib, A=(P[0], P[1], 48), M=5, K=40, W=(P[2], P[3], 64), N=24, bias=P[4], epi=0, gate=None, gs=24, rpb=2, out=P[6],
            ws=None, ws_bytes=0, dtype=BF16):
    a, w = (None if r is None else C.byref(_i8(lib, *r)) for r in (A, W))
    return lib.lib.orch_op_linear_quantized(a, M, K, w, N, bias, epi, gate, gs, rpb, out, ws, ws_bytes, dtype, None)


@pytest.mark.parametrize("kw,word", [
    (dict(dtype=-1), "dtype"), (dict(epi=3), "epilogue"), (dict(M=-1), "shape"), (dict(N=0), "shape"), (dict(K=0), "shape"),
    (dict(K=131072), "shape"), (dict(M=1 << 30, N=1 << 20), "too large"), (dict(M=(1 << 30) - 64, N=1), "too large"), (dict(A=None), "NULL"), (dict(W=None), "NULL"),
    (dict(A=(None, P[1], 48)), "NULL"), (dict(W=(P[2], None, 64)), "NULL"), (dict(A=(P[0] + 8, P[1], 48)), "16-byte"),
    (dict(A=(P[0], P[1], 32)), "multiple of 16"), (dict(W=(P[2], P[3], 56)), "multiple of 16"),
    (dict(W=(P[2], P[3], 1 << 23)), "2^23"), (dict(bias=P[4] + 2), "bias"), (dict(out=None), "NULL"),
    (dict(out=P[6] + 1), "aligned"), (dict(out=P[6] + 2, dtype=F32), "aligned"), (dict(out=P[6] + 2, epi=2, gate=P[5]), "aligned"),
    (dict(ws=P[7] + 4, ws_bytes=64), "workspace"), (dict(epi=2), "gate"), (dict(epi=2, gate=P[5], rpb=0), "rows_per_batch"),
    (dict(epi=2, gate=P[5], gs=23), "gate_stride"), (dict(epi=2, gate=P[5], gs=1 << 40), "gate_stride"),
    (dict(epi=2, gate=P[5] + 1), "gate"), (dict(out=P[0] + 16), "overlaps"), (dict(out=P[3]), "overlaps"),
    (dict(out=P[4] - 16), "overlaps"), (dict(epi=2, gate=P[6] + 32), "overlaps"), (dict(ws=P[0], ws_bytes=16), "overlaps"),
    (dict(ws=P[6] + 16, ws_bytes=16), "overlap"),
])
def test_linear_refuses(orch_lib, kw, word):
    _refused(orch_lib, _linear(orch_lib, **kw), word)


def _qkv(lib, A=(P[0], P[1], 48), B=2, n=5, K=40, W=(P[2], P[3], 48), bias=P[4], heads=2, d=32, q=P[6], kv=P[7], bs=2 * 9 * 64,
         tokens=9, off=4, ws=None, ws_bytes=0, dtype=BF16):
    a, w = (C.byref(_i8(lib, *r)) for r in (A, W))
    return lib.lib.orch_op_qkv_projection_quantized(a, B, n, K, w, bias, heads, d, q, kv, bs, tokens, off, ws, ws_bytes, dtype, None)


@pytest.mark.parametrize("kw,word", [
    (dict(d=48), "head_dim"), (dict(B=0), "shape"), (dict(n=-1), "shape"), (dict(heads=0), "shape"), (dict(heads=2048), "65536"),
    (dict(B=1 << 20, n=1 << 20), "shape"), (dict(off=5), "buffer"), (dict(off=-1), "buffer"), (dict(n=10), "buffer"),
    (dict(tokens=0, off=0, n=0), "buffer"), (dict(dtype=9), "dtype"), (dict(K=0), "shape"), (dict(q=None), "NULL"),
    (dict(kv=None), "NULL"), (dict(bs=2 * 9 * 64 - 8), "stride"), (dict(bs=1 << 40), "stride"), (dict(bs=2 * 9 * 64 + 4), "16-byte"),
    (dict(q=P[6] + 8), "16-byte"), (dict(kv=P[7] + 4), "16-byte"), (dict(q=P[0]), "overlaps"), (dict(kv=P[2] - 64), "overlaps"),
    (dict(q=P[7] + 64), "overlap"), (dict(ws=P[7], ws_bytes=64), "overlap"), (dict(A=(P[0], P[1], 32)), "multiple of 16"),
])
def test_qkv_refuses(orch_lib, kw, word):
    _refused(orch_lib, _qkv(orch_lib, **kw), word)


@pytest.mark.parametrize("shape", [(0, 8, 8), (8, 0, 8), (8, 8, 0), (8, 8, 131072), (-1, 8, 8), (1 << 30, 1 << 20, 8)])
def test_no_workspace_for_bad_shapes(orch_lib, shape):
    assert orch_lib.lib.orch_linear_quantized_workspace_bytes(*shape) == 0


def test_workspace_of_a_long_k_alone(orch_lib):
    """A projection's K needs none; a long one's k-splits hold an int32 for each output."""
    f = orch_lib.linear_quantized_workspace_bytes
    assert f(3328, 4608, 1152) == 0 and f(1, 1152, 4608) == 0
    assert f(32, 128, 18432) == 9 * 32 * 128 * 4


# ---- the binding -------------------------------------------------------------------

def _tensors(rows=4, cols=32):
    return torch.zeros((rows, cols), dtype=torch.int8), torch.zeros(rows)


def _raises(lib, word, f, *a, **kw):
    with pytest.raises(lib.OrchError) as e:
        f(*a, **kw)
    assert word in str(e.value), str(e.value)


def test_binding_of_int8_rows_refuses(orch_lib):
    lib = orch_lib
    v, s = _tensors()
    _raises(lib, "int8", lib.int8_rows, v.to(torch.uint8), s)
    _raises(lib, "fp32", lib.int8_rows, v, s.double())
    _raises(lib, "scales", lib.int8_rows, v, s[:3])
    _raises(lib, "scales", lib.int8_rows, v, torch.zeros(8)[::2])
    _raises(lib, "next to each other", lib.int8_rows, v.t(), torch.zeros(32))
    _raises(lib, "norm", lib.norm, "batch")
    _raises(lib, "weight", lib.norm, "rms", 1e-6, torch.zeros(4).double())
    _raises(lib, "weight", lib.norm, "rms", 1e-6, torch.zeros(8)[::2])
    _raises(lib, "weight", lib.norm, "layer", 1e-6, None, torch.zeros((2, 2)))


def test_binding_of_the_norms_refuses(orch_lib):
    lib = orch_lib
    h, y, m = torch.zeros((6, 32)), torch.zeros((6, 32), dtype=torch.bfloat16), torch.zeros((2, 32))
    f = lib.block_norms
    for kw in (dict(y=y[:5]), dict(y=y.half()), dict(h_out=y), dict(out=h, y=y), dict(out=torch.zeros((32, 6)).t()),
               dict(h_out=h[:, :16]), dict(gate=m.double(), rows_per_batch=3), dict(gate=m[:1], rows_per_batch=3),
               dict(gate=m, shift=torch.zeros((2, 40))[:, :32], rows_per_batch=3), dict(scale=m[:, :16], rows_per_batch=3),
               dict(out=lib.int8_rows(*_tensors(5))), dict(out=h, pre=lib.norm("rms", 1e-6, torch.zeros(16)))):
        with pytest.raises(lib.OrchError):
            f(h, **kw)
    with pytest.raises(lib.OrchError):
        f(y, None, None, h)
    _raises(lib, "int's range", f, h, None, h, gate=m, rows_per_batch=1 << 31)


def test_binding_of_the_products_refuses(orch_lib):
    lib = orch_lib
    A, W = lib.int8_rows(*_tensors(4)), lib.int8_rows(*_tensors(96))
    _raises(lib, "x must be", lib.quantize_rows, torch.zeros((4, 31)), A)
    _raises(lib, "x must be", lib.quantize_rows, torch.zeros((32, 4)).t(), A)
    _raises(lib, "type", lib.quantize_rows, torch.zeros((4, 32)).half(), A)
    out = torch.zeros((4, 96))
    f = lib.linear_quantized
    _raises(lib, "channels", f, A, lib.int8_rows(*_tensors(96, 48)), None, 0, out)
    _raises(lib, "bias", f, A, W, torch.zeros(95), 0, out)
    _raises(lib, "bias", f, A, W, torch.zeros(96).bfloat16(), 0, out)
    _raises(lib, "out must be", f, A, W, None, 0, torch.zeros((4, 95)))
    _raises(lib, "out must be", f, A, W, None, 0, torch.zeros((96, 4)).t())
    _raises(lib, "type", f, A, W, None, 0, out.half())
    _raises(lib, "workspace", f, A, W, None, 0, out, workspace=torch.zeros((4, 8))[:, ::2])
    _raises(lib, "adds to fp32", f, A, W, None, lib.EPI_RESIDUAL, out.bfloat16(), gate=torch.zeros((1, 96)), rows_per_batch=4)
    for g, rpb in ((None, 4), (torch.zeros((1, 96)), 3), (torch.zeros((2, 95)), 2), (torch.zeros((1, 96)).bfloat16(), 4)):
        _raises(lib, "gate", f, A, W, None, lib.EPI_RESIDUAL, out, gate=g, rows_per_batch=rpb)
    q, kv = torch.zeros((1, 1, 4, 32)), torch.zeros((1, 2 * 6 * 32))
    g = lib.qkv_projection_quantized
    _raises(lib, "q_out", g, A, W, None, q[:, :, :3], kv, 6, 0)
    _raises(lib, "q_out", g, A, W, None, torch.zeros((1, 2, 4, 32)), kv, 6, 0)
    _raises(lib, "kv_out", g, A, W, None, q, kv[0], 6, 0)
    _raises(lib, "kv_out", g, A, W, None, q, kv.bfloat16(), 6, 0)
    _raises(lib, "kv_out", g, A, W, None, q, kv, 7, 0)
    _raises(lib, "int's range", g, A, W, None, q, kv, 6, 1 << 31)
    _raises(lib, "int's range", lib.linear_quantized_workspace_bytes, 1 << 31, 1, 1)


def test_binding_refuses_the_host_and_other_gpus(orch_lib, monkeypatch):
    """Tensors that are not on the current GPU, and a stream of another one."""
    lib = orch_lib
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    A, W = lib.int8_rows(*_tensors(4)), lib.int8_rows(*_tensors(96))
    h = torch.zeros((4, 32))
    for f in (lambda: lib.block_norms(h, None, h), lambda: lib.quantize_rows(h, A),
              lambda: lib.linear_quantized(A, W, None, 0, torch.zeros((4, 96))),
              lambda: lib.qkv_projection_quantized(A, W, None, torch.zeros((1, 1, 4, 32)), torch.zeros((1, 2 * 4 * 32)), 4, 0)):
        _raises(lib, "the host", f)


def test_struct_layouts(orch_lib):
    lib = orch_lib
    assert C.sizeof(lib.BlockNorms) == lib._BLOCK_NORMS.size
    assert len(lib._NO_NORM.packed) == C.sizeof(lib.Norm) == 24
