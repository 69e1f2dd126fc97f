"""A whole block with norms around it and its projections in 8-bit integers: every call on
the results of the one before, against the oracle; captured, replayed, on two streams."""
import numpy as np
import pytest
import torch

from oracle import integer as oi
from tests._gpu_util import DEV, code, rel_l2, to_dev, to_host

pytestmark = pytest.mark.gpu

BF16 = "bf16"
B, N, HEADS, D, TOKENS, OFF, MLP = 2, 45, 2, 64, 70, 12, 320
H = HEADS * D


class Block:
    def __init__(self, lib, seed):
        rng = np.random.default_rng(seed)
        self.lib, M = lib, B * N
        self.h = to_dev(rng.standard_normal((M, H)))
        self.mod = to_dev(0.3 * rng.standard_normal((B, 6, H)))
        self.w, self.bias = {}, {}
        for name, (n, k) in dict(qkv=(3 * H, H), o=(H, H), fc1=(MLP, H), fc2=(H, MLP)).items():
            w = to_dev(rng.standard_normal((n, k)) / np.sqrt(k), BF16)
            self.w[name] = lib.int8_rows(torch.zeros((n, k), dtype=torch.int8, device=DEV), torch.zeros(n, device=DEV))
            lib.quantize_rows(w, self.w[name])                      # laid out once, as a program does
            self.bias[name] = to_dev(0.1 * rng.standard_normal(n))
        e = lambda *s: torch.empty(s, dtype=torch.bfloat16, device=DEV)
        self.q, self.kv, self.att = e(B, HEADS, N, D), to_dev(rng.standard_normal((B, 2 * TOKENS * H)), BF16), e(B * N, H)
        self.y1, self.f, self.y2 = e(M, H), e(M, MLP), e(M, H)
        self.h1, self.h2 = torch.empty((M, H), device=DEV), torch.empty((M, H), device=DEV)
        codes = lambda k: lib.int8_rows(torch.zeros((M, k), dtype=torch.int8, device=DEV), torch.zeros(M, device=DEV))
        self.u, self.a8, self.v, self.f8 = codes(H), codes(H), codes(H), codes(MLP)
        self.norm = {k: lib.norm(*v) for k, v in dict(pre=("layer", 1e-6), post=("rms", 1e-6)).items()}

    def run(self, stream=None):
        L, m, n, bias, w = self.lib, self.mod, self.norm, self.bias, self.w
        st = dict(stream=stream)
        L.block_norms(self.h, None, None, self.u, pre=n["pre"], shift=m[:, 0], scale=m[:, 1], rows_per_batch=N, **st)
        L.qkv_projection_quantized(self.u, w["qkv"], bias["qkv"], self.q, self.kv, TOKENS, OFF, **st)
        L.attention(self.q, self.kv, 2 * TOKENS * H, None, 0, 0, 0, B, HEADS, N, TOKENS, D, self.att, code(BF16), **st)
        L.quantize_rows(self.att, self.a8, **st)
        L.linear_quantized(self.a8, w["o"], bias["o"], L.EPI_STORE, self.y1, **st)
        L.block_norms(self.h, self.y1, self.h1, self.v, post=n["post"], pre=n["pre"], gate=m[:, 2], shift=m[:, 3],
                      scale=m[:, 4], rows_per_batch=N, **st)
        L.linear_quantized(self.v, w["fc1"], bias["fc1"], L.EPI_GELU, self.f, **st)
        L.quantize_rows(self.f, self.f8, **st)
        L.linear_quantized(self.f8, w["fc2"], bias["fc2"], L.EPI_STORE, self.y2, **st)
        L.block_norms(self.h1, self.y2, self.h2, None, post=n["post"], gate=m[:, 5], rows_per_batch=N, **st)

    def outputs(self):
        return [t.clone() for t in (self.q, self.kv, self.y1, self.h1, self.f, self.y2, self.h2, *self.u.tensors, *self.a8.tensors,
                                    *self.v.tensors, *self.f8.tensors)]


def _held(r):
    v, s = r.tensors
    return v.cpu().numpy(), s.cpu().numpy()


def test_block(orch_lib):
    b = Block(orch_lib, 0)
    kv0 = to_host(b.kv)
    b.run()
    torch.cuda.synchronize()
    m = to_host(b.mod)
    none, ln, rms = ("none", 0.0), ("layer", 1e-6), ("rms", 1e-6)
    # norms into codes: half a code off at most, beside what 32 bits lose: 48 roundings (2^-24) of a row's
    # largest value, which is five deviations, and six of the row itself: below 2e-5 of the largest output
    for codes, h, y, post, i in ((b.u, b.h, None, none, 0), (b.v, b.h, b.y1, rms, 3)):
        h1, u = oi.block_norms(to_host(h), None if y is None else to_host(y), post, ln, m[:, 2], m[:, i], m[:, i + 1], N)
        q, s = _held(codes)
        assert (np.abs(q * s[:, None].astype(np.float64) - u) <= s[:, None] * 0.5 + 2e-5 * np.abs(u).max(1, keepdims=True)).all()
    assert rel_l2(to_host(b.h1), h1) < 1e-6
    # products of the codes as they are: the output's rounding (2^-8 at most, each), and three of 32 bits
    # of sums that stay below 40: below 1e-5
    mm = lambda A, name: oi.product(*_held(A), *_held(b.w[name]), to_host(b.bias[name]))
    wq, wkv = oi.qkv(mm(b.u, "qkv"), B, HEADS, kv0, TOKENS, OFF)
    for got, want in ((b.q, wq), (b.kv, wkv), (b.y1, mm(b.a8, "o")), (b.f, oi.gelu_tanh(mm(b.v, "fc1"))), (b.y2, mm(b.f8, "fc2"))):
        g = to_host(got)
        assert (np.abs(g - want) <= 2.0 ** -8 * np.abs(want) + 1e-5).all()
    for codes, x in ((b.a8, b.att), (b.f8, b.f)):
        wq, ws = oi.quantize_rows(to_host(x))
        q, s = _held(codes)
        np.testing.assert_array_equal(q, wq)
        np.testing.assert_array_equal(s, ws)
    h2, _ = oi.block_norms(to_host(b.h1), to_host(b.y2), rms, none, m[:, 5], None, None, N)
    assert rel_l2(to_host(b.h2), h2) < 1e-6


def test_captured_and_replayed(orch_lib):
    """Replays follow what the inputs hold, with other work and synchronisations between them."""
    b, other = Block(orch_lib, 1), Block(orch_lib, 2)
    b.run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b.run()
    for i in range(4):
        h = to_dev(np.random.default_rng(10 + i).standard_normal((B * N, H)))
        b.h.copy_(h)
        b.run()
        want = b.outputs()
        for t in (b.y1, b.f, b.y2, b.h1, b.h2):
            t.zero_()
        other.run()                                     # the same kernels in between
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(b.outputs(), want):
            assert torch.equal(x, y)


def test_two_streams(orch_lib):
    """Two blocks at once, on streams of their own, by argument and as the current one."""
    blocks = [Block(orch_lib, s) for s in (3, 4)]
    want = []
    for b in blocks:
        b.run()
        want.append(b.outputs())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in blocks]
    for _ in range(5):
        for b, s in zip(blocks, streams):
            b.run(stream=s)
        with torch.cuda.stream(streams[0]):
            blocks[0].run()
    torch.cuda.synchronize()
    for b, w in zip(blocks, want):
        for x, y in zip(b.outputs(), w):
            assert torch.equal(x, y)


def test_large_offsets(orch_lib):
    """Rows whose outputs lie past 2^31 elements and 2^32 bytes."""
    lib = orch_lib
    M, K, n = 460000, 32, 4736                          # 2.18e9 outputs of bf16, 4.4 GB
    g = torch.Generator(device=DEV).manual_seed(0)
    a = torch.randint(-127, 128, (M, K), dtype=torch.int8, device=DEV, generator=g)
    w = torch.randint(-127, 128, (n, K), dtype=torch.int8, device=DEV, generator=g)
    sa, sw = torch.rand(M, device=DEV, generator=g), torch.rand(n, device=DEV, generator=g)
    out = torch.empty((M, n), dtype=torch.bfloat16, device=DEV)
    lib.linear_quantized(lib.int8_rows(a, sa), lib.int8_rows(w, sw), None, lib.EPI_STORE, out)
    rows = torch.tensor([0, 1, M // 2, 453437, 453438, M - 257, M - 1], device=DEV)
    want = oi.product(a[rows].cpu().numpy(), sa[rows].cpu().numpy(), w.cpu().numpy(), sw.cpu().numpy())
    got = to_host(out[rows])
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 3 * 2.0 ** -24 * np.abs(want)).all()
    # and through the quantiser and the norms, in place
    codes = lib.int8_rows(torch.empty((M, n), dtype=torch.int8, device=DEV), torch.empty(M, device=DEV))
    lib.quantize_rows(out, codes)
    wq, ws = oi.quantize_rows(got)
    np.testing.assert_array_equal(codes.tensors[0][rows].cpu().numpy(), wq)
    np.testing.assert_array_equal(codes.tensors[1][rows].cpu().numpy(), ws)
    h = torch.zeros((M, n), device=DEV)
    lib.block_norms(h, out, h, out, post=lib.norm("rms"), pre=lib.norm("layer"))
    h1, u = oi.block_norms(np.zeros_like(got), got, ("rms", 1e-6), ("layer", 1e-6))
    assert rel_l2(to_host(h[rows]), h1) < 1e-6
    assert (np.abs(to_host(out[rows]) - u) <= 2.0 ** -8 * np.abs(u) + 1e-5).all()
