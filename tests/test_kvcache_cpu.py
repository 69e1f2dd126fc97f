"""CPU side of the rotary positions, the 8-bit K/V cache and the attention over
it: the oracle's pins, and every call that the library refuses (checked before
anything is launched, so no GPU is needed; the pointers are never read)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import kvcache as ok
from tests import _attention_forms as forms

F32, BF16 = 0, 1
P = [0x10000000 * (i + 1) for i in range(8)]      # addresses far apart, 16-byte aligned


# ---- the oracle ------------------------------------------------------------------

def test_e4m3_table_is_torchs():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    np.testing.assert_array_equal(t, ok.e4m3_table())


def test_rounding_is_torchs():
    x = np.concatenate([np.linspace(-448, 448, 20001), np.linspace(-0.04, 0.04, 4001),
                        0.5 * (ok.e4m3_table()[:126] + ok.e4m3_table()[1:127])])
    x = x.astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(ok.to_e4m3(x.astype(np.float64)), want)


def test_scale_is_the_smallest():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((500, 8)) * 2.0 ** rng.integers(-140, 120, (500, 1))
    x[0], x[1] = 0.0, [448, 0, 0, 0, 0, 0, 0, -1]
    x[2] = np.nextafter(448, 500) * np.array([1, 0, 0, 0, 0, 0, 0, 0])
    v, e = ok.quantize(x)
    s, amax = 2.0 ** (e.astype(float) - 127), np.abs(x).max(-1)
    assert e.min() >= 1 and e[0] == 1 and e[1] == 127 and e[2] == 128
    assert (amax <= 448 * s).all() and ((amax > 224 * s) | (e == 1)).all()
    # half a step: 2^-4 of a value, 2^-10 s below the smallest normal 2^-6 s
    err = np.abs(ok.dequantize(v, e) - x)
    assert (err <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * s[:, None])).all()


def test_not_finite_is_nan_and_the_rest_keeps_its_scale():
    v, e = ok.quantize(np.array([[1.0, np.inf, -np.inf, np.nan]]))
    np.testing.assert_array_equal(ok.dequantize(v, e), [[1.0, np.nan, np.nan, np.nan]])


@pytest.mark.parametrize("interleaved", [True, False])
def test_rotation_depends_on_distance_alone(interleaved):
    """Scores of rotated q and k depend on the tokens' offset on the grid only."""
    rng = np.random.default_rng(1)
    q, k = (np.broadcast_to(rng.standard_normal((1, 1, 1, 32)), (1, 1, 64, 32)) for _ in range(2))
    rot = [ok.rotary(x, 0, (8, 10, 12), (4, 4, 4), (0.5, -3.0, 7.0), (1.0, 2.0, 0.5), 100.0, interleaved)[0, 0] for x in (q, k)]
    s = rot[0] @ rot[1].T
    tok = lambda f, r, c: (f * 4 + r) * 4 + c
    assert s[tok(0, 0, 0), tok(1, 2, 3)] == pytest.approx(s[tok(2, 1, 0), tok(3, 3, 3)], rel=1e-12)
    np.testing.assert_allclose((rot[0] ** 2).sum(-1), (q[0, 0] ** 2).sum(-1), rtol=1e-12)


# ---- refusals --------------------------------------------------------------------

def _refused(lib, rc, word):
    assert rc == lib.ORCH_EINVAL
    assert word in lib.last_error(), lib.last_error()


def _rotary(lib, tensors=None, n_tensors=1, B=1, n_tok=4, begin=0, d=32, dtype=BF16, **axes):
    ax = lib.rotary_axes(axes.get("channels", (0, 16, 16)), axes.get("extent", (1, 4, 4)), axes.get("theta", 1e4),
                         axes.get("origin", (0, 0, 0)), axes.get("step", (1, 1, 1)))
    if tensors is None:
        tensors = [dict()]
    ts = (lib.RotaryTensor * 2)()
    for t, kw in zip(ts, tensors):
        t.x, t.out, t.heads = kw.get("x", P[0]), kw.get("out", P[1]), kw.get("heads", 2)
        t.x_stride[:] = kw.get("xs", (2 * n_tok * d, n_tok * d, d))
        t.out_stride[:] = kw.get("os", (2 * n_tok * d, n_tok * d, d))
    return lib.lib.orch_op_rotary(C.byref(ax), ts, n_tensors, B, n_tok, begin, d, dtype, None)


@pytest.mark.parametrize("kw,word", [
    (dict(n_tensors=0), "n_tensors"), (dict(n_tensors=3), "n_tensors"), (dict(B=0), "B"), (dict(d=40), "head_dim"),
    (dict(dtype=2), "dtype"), (dict(theta=0.0), "theta"), (dict(theta=float("nan")), "theta"),
    (dict(channels=(0, 15, 16)), "channels"), (dict(channels=(2, 16, 16)), "channels"),
    (dict(channels=(-2, 16, 16)), "channels"), (dict(extent=(1, 0, 4)), "extents"),
    (dict(extent=(1 << 15, 1 << 15, 2)), "extents"), (dict(origin=(0, float("inf"), 0)), "origin"),
    (dict(step=(0, 0, float("nan"))), "step"), (dict(n_tok=17), "grid"), (dict(begin=13), "grid"),
    (dict(begin=-1), "grid"), (dict(n_tok=-1), "grid"), (dict(begin=2 ** 31 - 1), "grid"),
    (dict(extent=(1 << 10, 1 << 10, 1 << 10), n_tok=1 << 27), "2^31"),
    (dict(theta=1e-300, step=(1, 1, 1e50)), "angle"), (dict(origin=(0, 1e300, 0), step=(1, 1e300, 1)), "angle"),
    (dict(tensors=[dict(x=None)]), "NULL"), (dict(tensors=[dict(out=None)]), "NULL"),
    (dict(tensors=[dict(heads=0)]), "heads"), (dict(tensors=[dict(heads=40000)]), "heads"),
    (dict(tensors=[dict(x=P[0] + 1)]), "aligned"), (dict(tensors=[dict(xs=(0, 128, 31))]), "strides"),
    (dict(tensors=[dict(os=(0, 16, 32))]), "strides"), (dict(B=2, tensors=[dict(os=(8, 128, 32))]), "strides"),
    (dict(n_tensors=2, tensors=[dict(), dict(out=None)]), "NULL"),
    (dict(n_tensors=2, tensors=[dict(out=P[0]), dict(out=P[0])]), "overlap"),
    (dict(n_tensors=2, tensors=[dict(), dict(x=P[2], out=P[0])]), "overlap"),
    (dict(n_tensors=2, tensors=[dict(), dict(x=P[1], out=P[2])]), "overlap"),
])
def test_rotary_refuses(orch_lib, kw, word):
    _refused(orch_lib, _rotary(orch_lib, **kw), word)


def test_rotary_binding_refuses(orch_lib):
    ax = orch_lib.rotary_axes((0, 16, 16), (1, 4, 4))
    x = torch.zeros((1, 2, 4, 32))
    for a, b in ((x, x[..., :16]), (x, x.bfloat16()), (x.half(), x.half()), (x.transpose(2, 3), x.transpose(2, 3)),
                 ((x, x), (x,)), ((x, x[:, :, :2]), (x, x[:, :, :2]))):
        with pytest.raises(orch_lib.OrchError):
            orch_lib.rotary(ax, 0, a, b)


def _cache(lib, values=P[2], exponents=P[3], tokens=64, heads=2, d=32, vs=None, es=None):
    return lib.QuantizedKV(values, exponents, 2 * heads * tokens * d if vs is None else vs,
                           2 * heads * tokens if es is None else es, tokens)


COMMON = [
    (dict(B=0), "B"), (dict(heads=0), "heads"), (dict(B=200, heads=200), "heads"), (dict(d=40), "head_dim"),
    (dict(dtype=2), "dtype"), (dict(cache=dict(values=None)), "cache"), (dict(cache=dict(exponents=None)), "cache"),
    (dict(cache=dict(tokens=0)), "tokens"), (dict(cache=dict(tokens=1 << 26)), "2^31"),
    (dict(B=2, cache=dict(vs=16)), "stride"), (dict(B=2, cache=dict(es=16)), "stride"),
    (dict(cache=dict(values=P[2] + 8)), "aligned"), (dict(B=2, cache=dict(vs=1 << 20 | 8)), "aligned"),
    (dict(cache=dict(exponents=P[2] + 64)), "overlap"),
]
RANGES = [
    (dict(kv=None), "NULL"), (dict(n=-1), "tokens"), (dict(kv_off=-1), "tokens"), (dict(off=-1), "tokens"),
    (dict(n=41), "tokens"), (dict(n=40, off=25), "tokens"), (dict(kv_off=33), "tokens"),
    (dict(kv_off=2 ** 31 - 1), "tokens"), (dict(kv_tokens=0, n=0), "tokens"), (dict(kv_tokens=1 << 26), "2^31"),
    (dict(B=2, bs=16), "stride"), (dict(kv=P[0] + 2), "aligned"), (dict(B=2, bs=(1 << 20) + 4), "aligned"),
    (dict(kv=P[2] - 64), "overlap"), (dict(kv=P[3] - 64), "overlap"),
]


def _move(lib, back, kv=P[0], bs=1 << 20, kv_tokens=40, kv_off=0, off=0, B=1, heads=2, n=8, d=32, dtype=BF16, cache=None):
    c = _cache(lib, **(cache or {}))
    if back:
        return lib.lib.orch_op_kv_dequantize(C.byref(c), off, kv, bs, kv_tokens, kv_off, B, heads, n, d, dtype, None)
    return lib.lib.orch_op_kv_quantize(kv, bs, kv_tokens, kv_off, C.byref(c), off, B, heads, n, d, dtype, None)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("kw,word", COMMON + RANGES)
def test_cache_refuses(orch_lib, back, kw, word):
    _refused(orch_lib, _move(orch_lib, back, **kw), word)


def _attend(lib, q=P[0], fresh=P[1], bs=1 << 20, fb=4, nf=8, B=1, heads=2, n_q=8, d=32, out=P[4], ws=None, wsb=0,
            dtype=BF16, cache=None):
    c = _cache(lib, **(cache or {}))
    return lib.lib.orch_op_attention_quantized(q, C.byref(c), fresh, bs, fb, nf, B, heads, n_q, d, out, ws, wsb, dtype, None)


@pytest.mark.parametrize("kw,word", COMMON + [
    (dict(q=None), "NULL"), (dict(out=None), "NULL"), (dict(fresh=None), "NULL"), (dict(n_q=-1), "shape"),
    (dict(nf=-1), "shape"), (dict(fb=-1), "shape"), (dict(fb=57), "shape"), (dict(fb=2 ** 31 - 1), "shape"),
    (dict(B=2, bs=16), "stride"), (dict(q=P[0] + 2), "aligned"), (dict(out=P[4] + 4), "aligned"),
    (dict(fresh=P[1] + 8), "aligned"), (dict(B=2, bs=(1 << 20) + 4), "aligned"), (dict(ws=P[5] + 8, wsb=64), "aligned"),
    (dict(n_q=1 << 26), "2^31"), (dict(out=P[0]), "overlap"), (dict(out=P[2]), "overlap"), (dict(out=P[1]), "overlap"),
])
def test_attention_refuses(orch_lib, kw, word):
    _refused(orch_lib, _attend(orch_lib, **kw), word)


def test_null_cache_refused(orch_lib):
    _refused(orch_lib, orch_lib.lib.orch_op_kv_quantize(P[0], 1 << 20, 40, 0, None, 0, 1, 2, 8, 32, BF16, None), "cache")
    _refused(orch_lib, orch_lib.lib.orch_op_kv_dequantize(None, 0, P[0], 1 << 20, 40, 0, 1, 2, 8, 32, BF16, None), "cache")
    _refused(orch_lib, orch_lib.lib.orch_op_attention_quantized(P[0], None, None, 0, 0, 0, 1, 2, 8, 32, P[1], None, 0, BF16, None), "cache")


def test_binding_of_the_cache_refuses(orch_lib):
    v, e = torch.zeros((1, 2, 3, 8, 32), dtype=torch.uint8), torch.zeros((1, 2, 3, 8), dtype=torch.uint8)
    c = orch_lib.quantized_kv(v, e)
    assert (c.values, c.exponents, c.tokens) == (v.data_ptr(), e.data_ptr(), 8)
    for bad in ((v, e[..., :4]), (v.float(), e), (v, e.short()), (v[..., :16], e), (v[:, :1], e[:, :1]), (v.view(torch.float8_e5m2), e),
                (v.view(torch.float8_e4m3fnuz), e), (v.view(torch.int8), e), (v, e.view(torch.int8))):
        with pytest.raises(orch_lib.OrchError):
            orch_lib.quantized_kv(*bad)
    # a call of other branches, heads or channels than the cache's
    x = torch.zeros(4096, dtype=torch.bfloat16)
    for B, heads, d in ((2, 3, 32), (1, 2, 32), (1, 4, 32), (1, 3, 64)):
        for call in (lambda: orch_lib.kv_quantize(x, 0, 8, 0, c, 0, B, heads, 8, d, BF16),
                     lambda: orch_lib.kv_dequantize(c, 0, x, 0, 8, 0, B, heads, 8, d, BF16),
                     lambda: orch_lib.attention_quantized(x, c, None, 0, 0, 0, B, heads, 8, d, x, BF16)):
            with pytest.raises(orch_lib.OrchError, match="the cache holds"):
                call()


@pytest.mark.parametrize("bad", [dict(B=0), dict(heads=0), dict(n_q=-1), dict(n_kv=0), dict(d=0), dict(d=40), dict(dtype=7),
                                 dict(n_q=2 ** 31 - 1), dict(n_kv=2 ** 31 - 1), dict(n_q=1 << 25), dict(B=40000)])
def test_no_workspace_for_bad_shapes(orch_lib, bad):
    a = dict(B=1, heads=2, n_q=1, n_kv=4096, d=64, dtype=BF16) | bad
    assert orch_lib.attention_quantized_workspace_bytes(*a.values()) == 0


def _record(lib, kv=P[0], B=3, exponents=4096 * 2, stride=4096 * 2 + 256, bs=1 << 20, out=P[4], n=0):
    """Caches [values of a branch][its exponents] of 64 tokens, 2 heads of 32 (8192 + 256 bytes), called for no tokens."""
    c = dict(vs=stride, es=stride, exponents=P[2] + exponents)
    return [_move(lib, False, kv=kv, bs=bs, B=B, n=n, cache=c), _move(lib, True, kv=kv, bs=bs, B=B, n=n, cache=c),
            _attend(lib, B=B, n_q=n, fresh=kv, bs=bs, out=out, cache=c)]


def test_branches_may_lie_between_each_other(orch_lib):
    """Values and exponents of a branch in one record, records anywhere, K/V buffers between them: no byte is shared."""
    assert _record(orch_lib) == [0, 0, 0]
    assert _record(orch_lib, stride=1 << 20) == [0, 0, 0]
    assert _record(orch_lib, exponents=-256) == [0, 0, 0]                       # exponents first
    # K/V of 40 tokens (10240 bytes) behind each of the first branches' records
    assert _record(orch_lib, stride=1 << 16, kv=P[2] + 8448 + 64, bs=1 << 15) == [0, 0, 0]
    assert _record(orch_lib, stride=1 << 16, kv=P[2] + (1 << 16) - 10240, bs=1 << 15) == [0, 0, 0]


@pytest.mark.parametrize("kw", [
    dict(exponents=8192 - 16), dict(exponents=-240), dict(stride=1 << 16, exponents=(1 << 16) - 16),
    dict(stride=1 << 16, exponents=2 * (1 << 16) + 8191), dict(stride=1 << 16, exponents=-2 * (1 << 16) - 16),
])
def test_branches_that_share_bytes_are_refused(orch_lib, kw):
    for rc in _record(orch_lib, **kw):
        _refused(orch_lib, rc, "values and exponents overlap")


@pytest.mark.parametrize("at", [8448 - 16, -2 * 65536 + 8448 - 16, 2 * 65536 - 16, 65536 - 10240 + 16])
def test_buffers_that_share_bytes_with_a_branch_are_refused(orch_lib, at):
    """(At those places every other branch of the two is apart.)"""
    quantize, back, _ = _record(orch_lib, stride=1 << 16, kv=P[2] + at, bs=1 << 15)
    assert quantize == back == orch_lib.ORCH_EINVAL
    assert "overlap" in orch_lib.last_error()
    # the output of an attention (3 branches of 9 queries of 2 x 32 channels: 3456 bytes)
    c = dict(vs=1 << 16, es=1 << 16, exponents=P[2] + 8192)
    _refused(orch_lib, _attend(orch_lib, B=3, n_q=9, out=P[2] + 65536 + 8448 - 16, cache=c), "overlap")
    _refused(orch_lib, _attend(orch_lib, B=3, n_q=9, out=P[2] + 2 * 65536 - 3456 + 16, cache=c), "overlap")


def test_no_tokens_need_no_buffers(orch_lib):
    """An empty tensor has address 0: no tokens and no queries are no error, whatever the addresses."""
    assert _rotary(orch_lib, n_tok=0, tensors=[dict(x=None, out=None)]) == 0
    assert _rotary(orch_lib, n_tok=0, n_tensors=2, tensors=[dict(x=None, out=None), dict(x=None, out=None)]) == 0
    assert _attend(orch_lib, n_q=0, q=None, out=None) == 0
    assert _attend(orch_lib, n_q=0, q=None, out=None, fresh=None, fb=0, nf=0) == 0
    assert _move(orch_lib, False, n=0, kv=None) == 0 and _move(orch_lib, True, n=0, kv=None) == 0
    # the rest is checked all the same
    _refused(orch_lib, _rotary(orch_lib, n_tok=0, d=40, tensors=[dict(x=None, out=None)]), "head_dim")
    _refused(orch_lib, _attend(orch_lib, n_q=0, q=None, out=None, fresh=None), "NULL")
    _refused(orch_lib, _attend(orch_lib, n_q=0, q=None, out=None, cache=dict(values=None)), "cache")
    _refused(orch_lib, _move(orch_lib, True, n=0, kv=None, off=65), "tokens")


@pytest.mark.parametrize("kw", [
    dict(B=2, tensors=[dict(out=P[0], xs=(256, 128, 32), os=(512, 128, 32))]),
    dict(tensors=[dict(out=P[0], xs=(256, 128, 32), os=(256, 256, 32))]),
    dict(tensors=[dict(out=P[0], xs=(256, 128, 32), os=(256, 128, 64))]),
    dict(tensors=[dict(out=P[0], heads=4, xs=(512, 128, 32), os=(512, 32, 128))]),        # a transpose
    dict(n_tensors=2, tensors=[dict(), dict(x=P[2], out=P[2], os=(256, 256, 32))]),
])
def test_in_place_needs_the_same_strides(orch_lib, kw):
    _refused(orch_lib, _rotary(orch_lib, **kw), "in place")


def _bound(lib, kv=None, q=None, out=None, fresh=None, ws=None, dtype=BF16, bs=2 * 8 * 96, tokens=8, n_q=5, B=2):
    """The binding's three calls on host tensors (refused for that if for nothing else): 2 branches of 3 heads of 32."""
    t = torch.bfloat16
    cache = lib.quantized_kv(torch.zeros((2, 2, 3, 16, 32), dtype=torch.uint8), torch.zeros((2, 2, 3, 16), dtype=torch.uint8))
    kv = torch.zeros((2, 2 * 8 * 96), dtype=t) if kv is None else kv
    fresh = torch.zeros((2, 2 * 8 * 96), dtype=t) if fresh is None else fresh
    q = torch.zeros((2, 3, 5, 32), dtype=t) if q is None else q
    out = torch.zeros((2, 5, 96), dtype=t) if out is None else out
    return (lambda: lib.kv_quantize(kv, bs, tokens, 0, cache, 0, B, 3, 8, 32, dtype),
            lambda: lib.kv_dequantize(cache, 0, kv, bs, tokens, 0, B, 3, 8, 32, dtype),
            lambda: lib.attention_quantized(q, cache, fresh, bs, 0, tokens, B, 3, n_q, 32, out, dtype, workspace=ws))


ROWS = torch.zeros((2, 2 * 8 * 96 + 32), dtype=torch.bfloat16)
REFUSED_BUFFERS = [      # calls, arguments, message
    ((0, 1), dict(kv=torch.zeros((2, 2 * 8 * 96))), "type"), ((0, 1, 2), dict(dtype=F32), "type"),
    ((0, 1), dict(kv=torch.zeros((2, 2 * 8 * 96), dtype=torch.half)), "type"),
    ((0, 1), dict(kv=torch.zeros(2 * 2 * 8 * 96 - 1, dtype=torch.bfloat16)), "holds"),
    ((0, 1), dict(tokens=9), "holds"), ((0, 1, 2), dict(bs=2 * 8 * 96 + 8), "holds"), ((2,), dict(tokens=9), "holds"),
    ((0, 1), dict(kv=ROWS[:, :2 * 8 * 96]), "contiguous"), ((0, 1), dict(kv=torch.zeros((2, 8 * 96, 4), dtype=torch.bfloat16)[..., ::2]), "contiguous"),
    ((2,), dict(fresh=ROWS[:, :2 * 8 * 96]), "contiguous"), ((2,), dict(fresh=torch.zeros((2, 2 * 8 * 96))), "type"),
    ((2,), dict(q=torch.zeros((2, 3, 4, 32), dtype=torch.bfloat16)), "q holds"), ((2,), dict(n_q=6), "holds"),
    ((2,), dict(q=torch.zeros((2, 5, 3, 32), dtype=torch.bfloat16).transpose(1, 2)), "q must be contiguous"),
    ((2,), dict(q=torch.zeros((2, 3, 5, 32))), "q is"), ((2,), dict(out=torch.zeros((2, 5, 96))), "out is"),
    ((2,), dict(out=torch.zeros((2, 4, 96), dtype=torch.bfloat16)), "out holds"),
    ((2,), dict(out=torch.zeros((5, 2, 96), dtype=torch.bfloat16).transpose(0, 1)), "out must be contiguous"),
    ((2,), dict(ws=torch.zeros((64, 64), dtype=torch.uint8).t()[:, :3]), "workspace must be contiguous"),
]


@pytest.mark.parametrize("i", range(len(REFUSED_BUFFERS)))
def test_binding_refuses_buffers(orch_lib, i):
    """Tensors of another type than the code's, too small for the extents, or with other strides than the kernels read."""
    calls, kw, word = REFUSED_BUFFERS[i]
    for c in calls:
        with pytest.raises(orch_lib.OrchError, match=word):
            _bound(orch_lib, **kw)[c]()


@pytest.mark.parametrize("kw", [dict(), dict(kv=ROWS[:, :2 * 8 * 96], fresh=ROWS[:, :2 * 8 * 96], bs=2 * 8 * 96 + 32),
                                dict(kv=ROWS.view(-1), fresh=ROWS.view(-1)), dict(B=1, bs=0), dict(out=ROWS, q=ROWS)])
def test_binding_takes_buffers(orch_lib, monkeypatch, kw):
    """What they hold is enough: the next check, of the devices, is reached."""
    class Reached(Exception):
        pass

    def on(*_):
        raise Reached

    monkeypatch.setattr(orch_lib, "_stream_on", on)
    for call in _bound(orch_lib, **kw):
        with pytest.raises(Reached):
            call()


@pytest.mark.parametrize("d", forms.SIZES)
@pytest.mark.parametrize("form", forms.FORMS, ids=str)
def test_every_form_of_the_attention_has_a_shape(orch_lib, form, d):
    """What the GPU tests of the forms run; a shape with a workspace a byte short runs as without one."""
    assert forms.shape_for(orch_lib, form, d) is not None
    for shape in forms.CANDIDATES:
        a = (*shape, d, forms.CODE[form[0]])
        need = orch_lib.attention_quantized_workspace_bytes(*a)
        prepared, _, parts = whole = orch_lib.attention_quantized_plan(*a, need)
        without = orch_lib.attention_quantized_plan(*a, 0)
        assert (need > 0) == (prepared or parts > 1) and not without[0] and without[2] == 1
        assert orch_lib.attention_quantized_plan(*a, need + 1) == whole
        if need:
            assert orch_lib.attention_quantized_plan(*a, need - 1) == without


@pytest.mark.parametrize("bad", [dict(B=0), dict(heads=0), dict(n_q=0), dict(n_kv=0), dict(d=40), dict(dtype=7), dict(n_q=1 << 25),
                                 dict(B=40000)])
def test_no_plan_for_bad_shapes(orch_lib, bad):
    a = dict(B=1, heads=2, n_q=1, n_kv=4096, d=64, dtype=BF16) | bad
    with pytest.raises(orch_lib.OrchError, match="shape"):
        orch_lib.attention_quantized_plan(*a.values(), 0)
    assert orch_lib.lib.orch_attention_quantized_plan(1, 2, 1, 4096, 64, BF16, 0, None, None, None) == orch_lib.ORCH_EINVAL


@pytest.mark.parametrize("big", [2 ** 31, 2 ** 32, 2 ** 32 + 4, -2 ** 31 - 1, -2 ** 32, 2 ** 64])
def test_binding_refuses_what_a_c_int_does_not_hold(orch_lib, monkeypatch, big):
    """ctypes would wrap it: 2^32 + 4 would be token 4."""
    class Reached(Exception):
        pass

    def on(*_):
        raise Reached

    monkeypatch.setattr(orch_lib, "_stream_on", on)
    x = torch.zeros((1, 2, 4, 32))
    for axes in (dict(extent=(1, 4, big)), dict(extent=(big, 1, 4)), dict(channels=(0, big, 16))):
        with pytest.raises(orch_lib.OrchError, match="int"):
            orch_lib.rotary_axes(**(dict(channels=(0, 16, 16), extent=(1, 4, 4)) | axes))
    with pytest.raises(orch_lib.OrchError, match="int"):
        orch_lib.rotary(orch_lib.rotary_axes((0, 16, 16), (1, 4, 4)), big, x, x)
    cache = orch_lib.quantized_kv(torch.zeros((1, 2, 2, 8, 32), dtype=torch.uint8), torch.zeros((1, 2, 2, 8), dtype=torch.uint8))
    kv, q, out = torch.zeros(2 * 8 * 64), torch.zeros((1, 2, 4, 32)), torch.zeros((1, 4, 64))
    for kv_off, off, n in ((big, 0, 4), (0, big, 4), (0, 0, big)):
        with pytest.raises(orch_lib.OrchError, match="int"):
            orch_lib.kv_quantize(kv, 0, 8, kv_off, cache, off, 1, 2, n, 32, F32)
        with pytest.raises(orch_lib.OrchError, match="int"):
            orch_lib.kv_dequantize(cache, off, kv, 0, 8, kv_off, 1, 2, n, 32, F32)
    for fb, nf, n_q in ((big, 4, 4), (0, 4, big), (0, big, 4)):
        with pytest.raises(orch_lib.OrchError, match="int|holds"):
            orch_lib.attention_quantized(q, cache, kv, 0, fb, nf, 1, 2, n_q, 32, out, F32)
    for call in (lambda: orch_lib.kv_quantize(kv, 0, 8, 2, cache, 3, 1, 2, 4, 32, F32),
                 lambda: orch_lib.attention_quantized(q, cache, kv, 0, 4, 4, 1, 2, 4, 32, out, F32)):
        with pytest.raises(Reached):
            call()


@pytest.mark.parametrize("stride", [2 ** 40, 2 ** 63, 2 ** 64 - 16 * 1024, 2 ** 61 + 2048, 2 ** 62 + 4096])
def test_strides_that_wrap_are_refused(orch_lib, stride):
    """No branch lies 2^40 away; past 2^61 or so the offsets would wrap, before the buffer's start too."""
    for back in (False, True):
        _refused(orch_lib, _move(orch_lib, back, B=2, bs=stride), "stride")
        for c in (dict(vs=stride), dict(es=stride)):
            _refused(orch_lib, _move(orch_lib, back, B=2, cache=c), "stride")
    _refused(orch_lib, _attend(orch_lib, B=2, bs=stride), "stride")
    _refused(orch_lib, _attend(orch_lib, B=2, cache=dict(vs=stride)), "stride")
    for a in range(3):
        xs = [256, 128, 32]
        xs[a] = stride
        _refused(orch_lib, _rotary(orch_lib, B=2, tensors=[dict(xs=xs)]), "strides")
        _refused(orch_lib, _rotary(orch_lib, B=2, tensors=[dict(os=xs)]), "strides")


def test_negative_branch_strides_are_refused(orch_lib):
    for call in _bound(orch_lib, bs=-2 * 8 * 96):
        with pytest.raises(orch_lib.OrchError, match="stride"):
            call()


def test_binding_refuses_a_stream_of_another_gpu(orch_lib, monkeypatch):
    class Stream:
        cuda_stream = 7

        def __init__(self, device):
            self.device_index = device

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    assert orch_lib._stream_on(Stream(0), 0, 0) == 7
    for stream, device in ((Stream(1), 0), (Stream(0), 1), (Stream(1), 1), (Stream(0), -1)):
        with pytest.raises(orch_lib.OrchError, match="current GPU"):
            orch_lib._stream_on(stream, device)


def test_binding_without_a_tensor(orch_lib, monkeypatch):
    """None is the library's to refuse, as a NULL pointer."""
    monkeypatch.setattr(orch_lib, "_stream_on", lambda *_: 0)
    cache = orch_lib.quantized_kv(torch.zeros((1, 2, 2, 8, 32), dtype=torch.uint8), torch.zeros((1, 2, 2, 8), dtype=torch.uint8))
    x = torch.zeros((1, 2, 4, 32))
    for q, out, fresh in ((None, x, x), (x, None, x), (x, x, None)):
        with pytest.raises(orch_lib.OrchError, match="NULL"):
            orch_lib.attention_quantized(q, cache, fresh, 0, 0, 1, 1, 2, 4, 32, out, F32)
