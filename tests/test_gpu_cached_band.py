"""The operators around the 8-bit cache together, as a band's attention layer uses them, eager, on another stream and
captured into graphs: QKV projection, rotary positions of Q and of K in the band's K/V buffer, attention over fresh +
cached K/V, the band written into the cache, and the whole cache read back into the buffer that orch_op_attention takes.
Each step is compared with the float64 oracle on the values that the step before left on the GPU."""
import numpy as np
import pytest
import torch

from oracle import kvcache as ok
from tests._gpu_util import DEV, code, empty, rounded, to_dev, to_host
from tests.test_gpu_attention_quantized import check as check_attention
from tests.test_gpu_rotary import _check as check_rotary

pytestmark = pytest.mark.gpu


class Band:
    """One layer's buffers for bands of an R x C image, B branches."""

    def __init__(self, lib, dtype, B, heads, d, R, C, seed):
        self.lib, self.dtype, self.B, self.heads, self.d, self.R, self.C = lib, dtype, B, heads, d, R, C
        self.N, self.H = R * C, heads * d
        self.rng = np.random.default_rng(seed)
        self.values = torch.zeros((B, 2, heads, self.N, d), dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
        self.exps = torch.full((B, 2, heads, self.N), 127, dtype=torch.uint8, device=DEV)
        self.cache = lib.quantized_kv(self.values, self.exps)
        self.W = to_dev(self.rng.standard_normal((3 * self.H, self.H)) / np.sqrt(self.H), dtype)
        self.bias = to_dev(self.rng.standard_normal(3 * self.H) * 0.1)
        # 4 channels pass, the rest for height and width
        h = (d - 4) // 4 * 2
        self.ch = (0, h, d - 4 - h)
        self.axes = lib.rotary_axes(self.ch, (1, R, C), 1e4, (0.0, -0.5 * R, -0.5 * C))

    def inputs(self, rows):
        return to_dev(self.rng.standard_normal((self.B * rows * self.C, self.H)), self.dtype)

    def buffers(self, rows):
        n = rows * self.C
        need = self.lib.attention_quantized_workspace_bytes(self.B, self.heads, n, self.N, self.d, code(self.dtype))
        return (empty((self.B, self.heads, n, self.d), self.dtype), empty((self.B, 2 * n * self.H), self.dtype),
                empty((self.B, n, self.H), self.dtype), torch.empty(max(need, 16), dtype=torch.uint8, device=DEV))

    def project(self, A, rows, q, kv):
        n = rows * self.C
        self.lib.qkv_projection(A, self.B, n, self.H, self.W, self.bias, self.H, self.heads, q, kv, 2 * n * self.H, n, 0,
                                code(self.dtype))

    def k_of(self, kv, n):
        return kv[:, :n * self.H].view(self.B, self.heads, n, self.d)

    def layer(self, A, row, rows, q, kv, out, ws):
        """The band [row, row + rows): its attention, then its K/V into the cache."""
        n, fb, c = rows * self.C, row * self.C, code(self.dtype)
        self.project(A, rows, q, kv)
        k = self.k_of(kv, n)
        self.lib.rotary(self.axes, fb, (q, k), (q, k))
        self.lib.attention_quantized(q, self.cache, kv, 2 * n * self.H, fb, n, self.B, self.heads, n, self.d, out, c, workspace=ws)
        self.lib.kv_quantize(kv, 2 * n * self.H, n, 0, self.cache, fb, self.B, self.heads, n, self.d, c)

    def cached(self):
        """The values that the cache stands for, [B, 2, heads, N, d]."""
        torch.cuda.synchronize()
        return ok.dequantize(self.values.view(torch.uint8).cpu().numpy(), self.exps.cpu().numpy())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,d,R,C,rows", [(4, 32, 8, 8, 4), (6, 64, 9, 15, 4), (4, 72, 16, 16, 6), (2, 128, 5, 13, 2)])
def test_layer_by_layer(orch_lib, dtype, heads, d, R, C, rows):
    x = Band(orch_lib, dtype, 2, heads, d, R, C, R + d)
    tok = {}
    for row in list(range(0, R - rows + 1, rows)) + [1]:          # every band, then one across two of them
        n, fb = rows * C, row * C
        A, (q, kv, out, ws) = x.inputs(rows), x.buffers(rows)
        x.project(A, rows, q, kv)
        q0, k0 = to_host(q), to_host(x.k_of(kv, n))
        before = x.cached()
        x.layer(A, row, rows, q, kv, out, ws)
        q1 = to_host(q)
        k1, v1 = ok.from_buffer(to_host(kv), heads, n, d)
        for got, src in ((q1, q0), (k1, k0)):
            check_rotary(got, src, ok.rotary(src, fb, x.ch, (1, R, C), (0, -0.5 * R, -0.5 * C), (1, 1, 1), 1e4, True), dtype)
        K, V = before[:, 0].copy(), before[:, 1].copy()
        K[:, :, fb:fb + n], V[:, :, fb:fb + n] = k1, v1
        check_attention(to_host(out).reshape(2, n, heads, d).transpose(0, 2, 1, 3), dtype, q1, K, V)
        after = x.cached()
        for i, y in enumerate((k1, v1)):
            before[:, i, :, fb:fb + n] = ok.dequantize(*ok.quantize(y))
        np.testing.assert_array_equal(after, before)
    # the whole image read back: what orch_op_attention takes, no fresh keys
    stale = empty((2, 2 * x.N * x.H), dtype)
    x.lib.kv_dequantize(x.cache, 0, stale, 2 * x.N * x.H, x.N, 0, 2, heads, x.N, d, code(dtype))
    K, V = ok.from_buffer(to_host(stale), heads, x.N, d)
    np.testing.assert_array_equal(np.stack((K, V), 1), x.cached())
    o2 = empty((2, n, x.H), dtype)
    x.lib.attention(q, stale, 2 * x.N * x.H, None, 0, 0, 0, 2, heads, n, x.N, d, o2, code(dtype))
    o3 = empty((2, n, x.H), dtype)
    x.lib.attention_quantized(q, x.cache, None, 0, 0, 0, 2, heads, n, d, o3, code(dtype), workspace=ws)
    for o in (o2, o3):
        got = to_host(o).reshape(2, n, heads, d).transpose(0, 2, 1, 3)
        ref = ok.attention(q1, K, V)
        assert np.linalg.norm(got - ref) <= (1e-2 if dtype == "bf16" else 2e-5) * np.linalg.norm(ref)


@pytest.mark.parametrize("dtype,heads,d,rows", [("bf16", 6, 64, 6), ("bf16", 16, 72, 32), ("f32", 4, 32, 4)])
def test_streams_and_graphs(orch_lib, dtype, heads, d, rows):
    """The same bits eager, on a stream of its own, and from two captured graphs that share nothing but the cache,
    replayed in turn with eager work between."""
    R, C = 64 if rows == 32 else 16, 64 if rows == 32 else 16
    x = Band(orch_lib, dtype, 2, heads, d, R, C, 7)
    A0 = x.inputs(R)
    b0 = x.buffers(R)
    x.layer(A0, 0, R, *b0)                                        # fill the cache
    start = (x.values.clone(), x.exps.clone())

    def restore():
        x.values.copy_(start[0])
        x.exps.copy_(start[1])

    bands = [(x.inputs(rows), row, x.buffers(rows)) for row in (0, R - rows)]

    def result():
        torch.cuda.synchronize()
        return [b[2][2].clone() for b in bands] + [x.values.view(torch.uint8).clone(), x.exps.clone()]

    def eager():
        restore()
        for A, row, b in bands:
            x.layer(A, row, rows, *b)
        return result()

    want = eager()
    side = torch.cuda.Stream()
    restore()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for A, row, b in bands:
            x.layer(A, row, rows, *b)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(result(), want))

    graphs = []
    for A, row, b in bands:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x.layer(A, row, rows, *b)
        graphs.append(g)
    for k in range(4):
        for A, row, b in bands:
            b[2].zero_()
        restore()
        for g in graphs:
            g.replay()
        got = result()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k
        if k == 1:
            assert all(torch.equal(a, b) for a, b in zip(eager(), want))


def test_two_streams_at_once(orch_lib):
    """Two attentions over one cache at the same time, each with a workspace of its own."""
    x = Band(orch_lib, "bf16", 2, 16, 72, 32, 32, 3)
    b0 = x.buffers(32)
    x.layer(x.inputs(32), 0, 32, *b0)
    calls = []
    for rows in (2, 30):
        n = rows * 32
        q, kv, out, ws = x.buffers(rows)
        x.project(x.inputs(rows), rows, q, kv)
        calls.append((rows, n, q, kv, out, ws))

    def call(c):
        rows, n, q, kv, out, ws = c
        x.lib.attention_quantized(q, x.cache, kv, 2 * n * x.H, 32, n, 2, 16, n, 72, out, 1, workspace=ws)

    for c in calls:
        call(c)
    torch.cuda.synchronize()
    want = [c[4].clone() for c in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for c, s in zip(calls, streams):
            with torch.cuda.stream(s):
                c[4].zero_()
                call(c)
    torch.cuda.synchronize()
    assert all(torch.equal(c[4], w) for c, w in zip(calls, want))


def test_host_tensors_are_refused(orch_lib):
    x = Band(orch_lib, "bf16", 1, 2, 32, 4, 4, 1)
    q, kv, out, ws = x.buffers(2)
    host = torch.zeros_like(kv, device="cpu")
    with pytest.raises(orch_lib.OrchError):
        orch_lib.kv_quantize(host, 2 * 8 * 64, 8, 0, x.cache, 0, 1, 2, 8, 32, 1)
    with pytest.raises(orch_lib.OrchError):
        orch_lib.kv_dequantize(x.cache, 0, host, 2 * 8 * 64, 8, 0, 1, 2, 8, 32, 1)
    with pytest.raises(orch_lib.OrchError):
        orch_lib.attention_quantized(q.cpu(), x.cache, kv, 0, 0, 8, 1, 2, 8, 32, out, 1)
    with pytest.raises(orch_lib.OrchError):
        orch_lib.rotary(x.axes, 0, q.cpu(), q)
    with pytest.raises(orch_lib.OrchError):
        orch_lib.kv_quantize(kv, 0, 8, 0, orch_lib.quantized_kv(x.values.cpu(), x.exps), 0, 1, 2, 8, 32, 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_an_empty_band(orch_lib, dtype):
    """No tokens, in torch's empty tensors (address 0): nothing is done, and the cache stays as it was."""
    x = Band(orch_lib, dtype, 2, 2, 32, 4, 4, 1)
    before = x.values.view(torch.uint8).clone()
    q, out, none = empty((2, 2, 0, 32), dtype), empty((2, 0, 64), dtype), empty((2, 0), dtype)
    assert q.data_ptr() == 0
    orch_lib.rotary(x.axes, 3, (q, q), (q, q.clone()))
    orch_lib.rotary(x.axes, 16, q, q)
    for fresh in (None, none):
        orch_lib.attention_quantized(q, x.cache, fresh, 0, 5, 0, 2, 2, 0, 32, out, code(dtype))
    orch_lib.kv_quantize(empty((2, 8 * 128), dtype), 8 * 128, 8, 3, x.cache, 5, 2, 2, 0, 32, code(dtype))
    torch.cuda.synchronize()
    assert torch.equal(before, x.values.view(torch.uint8))


def test_a_stream_given(orch_lib):
    """The stream argument: the same bits as on the current stream."""
    x = Band(orch_lib, "bf16", 2, 4, 72, 8, 8, 5)
    q, kv, _, ws = x.buffers(3)
    x.project(x.inputs(3), 3, q, kv)
    torch.cuda.synchronize()
    results = []
    for stream in (None, torch.cuda.Stream()):
        qo, out, back = torch.zeros_like(q), empty((2, 24, x.H), "bf16"), torch.zeros_like(kv)
        torch.cuda.synchronize()
        orch_lib.rotary(x.axes, 8, q, qo, stream=stream)
        orch_lib.kv_quantize(kv, 2 * 24 * x.H, 24, 0, x.cache, 8, 2, 4, 24, 72, 1, stream=stream)
        orch_lib.attention_quantized(qo, x.cache, kv, 2 * 24 * x.H, 8, 24, 2, 4, 24, 72, out, 1, workspace=ws, stream=stream)
        orch_lib.kv_dequantize(x.cache, 8, back, 2 * 24 * x.H, 24, 0, 2, 4, 24, 72, 1, stream=stream)
        torch.cuda.synchronize()
        results.append((qo, out, back))
    assert all(torch.equal(a, b) for a, b in zip(*results))
