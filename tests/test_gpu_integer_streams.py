"""A whole block of norms and 8-bit integer products in graphs and on streams, where every
intermediate and output is overwritten before each run: what does not run, or runs too early, shows."""
import numpy as np
import pytest
import torch

from tests._gpu_util import DEV, to_dev
from tests.test_gpu_integer_block import B, D, H, HEADS, N, OFF, TOKENS, Block

pytestmark = pytest.mark.gpu


def _band(b):
    """The band's K and V in the block's K/V buffer."""
    k, v = b.kv[:, :TOKENS * H].view(B, HEADS, TOKENS, D), b.kv[:, TOKENS * H:].view(B, HEADS, D, TOKENS)
    return k[:, :, OFF:OFF + N], v[..., OFF:OFF + N]


def _wipe(b):
    """NaN, and codes that no row has, in all that a run writes."""
    for t in (b.q, *_band(b), b.att, b.y1, b.f, b.y2, b.h1, b.h2):
        t.fill_(float("nan"))
    for r in (b.u, b.a8, b.v, b.f8):
        values, scales = r.tensors
        values.fill_(-128)
        scales.fill_(float("nan"))


def _outputs(b):
    return [b.att.clone(), *b.outputs()]


def _inputs(b, seed):
    b.h.copy_(to_dev(np.random.default_rng(seed).standard_normal((B * N, H))))


def _expected(b):
    """By a run of its own, on the default stream."""
    _wipe(b)
    b.run()
    want = _outputs(b)
    torch.cuda.synchronize()
    assert all(bool(torch.isfinite(t).all()) for t in want)
    return want


def _same(b, want):
    for i, (x, y) in enumerate(zip(_outputs(b), want)):
        assert torch.equal(x, y), i


def _capture(b):
    b.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        b.run()
    return graph


def test_replays_write_everything(orch_lib):
    b, other = Block(orch_lib, 11), Block(orch_lib, 12)
    graph = _capture(b)
    for i in range(4):
        _inputs(b, 20 + i)
        want = _expected(b)
        _wipe(b)
        other.run()                                     # the same kernels in between
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        _same(b, want)


def test_streams_write_everything(orch_lib):
    """Two blocks at once, new inputs each time, on streams by argument and as the current one."""
    blocks, streams = [Block(orch_lib, s) for s in (13, 14)], [torch.cuda.Stream() for _ in range(2)]
    for i in range(6):
        want = []
        for k, b in enumerate(blocks):
            _inputs(b, 40 + 2 * i + k)
            want.append(_expected(b))
            _wipe(b)
        torch.cuda.synchronize()
        for b, s in zip(blocks, streams):
            if i % 2:
                with torch.cuda.stream(s):
                    b.run()
            else:
                b.run(stream=s)
        torch.cuda.synchronize()
        for b, w in zip(blocks, want):
            _same(b, w)


def test_graphs_at_once(orch_lib):
    """Two graphs replayed on streams of their own, and a third block between them."""
    blocks, streams = [Block(orch_lib, s) for s in (15, 16)], [torch.cuda.Stream() for _ in range(2)]
    other, graphs = Block(orch_lib, 17), [_capture(b) for b in blocks]
    for i in range(4):
        want = []
        for k, b in enumerate(blocks):
            _inputs(b, 60 + 2 * i + k)
            want.append(_expected(b))
            _wipe(b)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
            other.run()
        torch.cuda.synchronize()
        for b, w in zip(blocks, want):
            _same(b, w)
