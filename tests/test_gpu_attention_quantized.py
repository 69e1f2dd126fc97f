"""Attention over fresh K/V and the 8-bit cache against the float64 oracle on the values that the cache stands for.

Tolerance, elementwise, with A = sum_n p_n |v_n| of the output's query and channel and S = the
largest sum of |q_c k_c| / sqrt(d) of a query:
  fp32  a score's rounding is at most (d + 2) 2^-24 S, a probability's twice that
        relative to the sum, the exponent's argument and the exponential 2^-21, and the sums of n products
        n 2^-24: A (2^-22 (d + 2) S + 2^-20 + n 2^-23).
  bf16  the same, a probability and the output rounded to bf16 once each (half a step, 2^-8), the
        sum of the rounded or the unrounded probabilities: A 2^-7 and 2^-8 |o| more.
"""
import numpy as np
import pytest
import torch

from oracle import kvcache as ok
from tests._gpu_util import DEV, code, rel_l2, rounded, to_dev, to_host

pytestmark = pytest.mark.gpu


# 2-norms.  A rounding to bf16 is off by at most 2^-8 of the value, evenly spread: 2^-8 / sqrt(3) = 2.26e-3 in
# the 2-norm where every value lies just above a power of two (half that just below one: 1.7e-3 over many).  A
# single query's few large probabilities may all lie there, and its outputs too: two independent roundings,
# sqrt(2) 2.26e-3 = 3.2e-3.
NORM = {"bf16": 3.2e-3, "f32": 1e-5}


def make(rng, dtype, B, heads, d, n_q, N, fb, nf, ramp=0.0, shift=0.0):
    """q, cache bytes, fresh K/V and the K/V that the attention stands for."""
    q = rng.standard_normal((B, heads, n_q, d))
    k, v = (rng.standard_normal((B, heads, N, d)) * 2.0 ** rng.integers(-2, 3, (B, heads, N, 1)) for _ in range(2))
    k *= 0.5
    fk, fv = (rng.standard_normal((B, heads, nf, d)) for _ in range(2))
    if ramp:
        k *= (1.0 + ramp * np.arange(N) / N)[None, None, :, None]
    if shift:
        q[..., 0] = k[..., 0] = fk[..., 0] = shift
    q, fk, fv = (rounded(x, dtype) for x in (q, fk, fv))
    (kv8, ke), (vv8, ve) = ok.quantize(k), ok.quantize(v)
    K, V = ok.dequantize(kv8, ke), ok.dequantize(vv8, ve)
    K[:, :, fb:fb + nf], V[:, :, fb:fb + nf] = fk, fv
    return q, np.stack((kv8, vv8), 1), np.stack((ke, ve), 1), fk, fv, K, V


def run(lib, dtype, q, v8, e8, fk, fv, fb, split=True, garbage=True):
    """The call on device copies.  The cache's bytes of the fresh tokens are NaN: never to be read."""
    B, heads, n_q, d = q.shape
    N, nf = v8.shape[3], fk.shape[2]
    v8, e8 = v8.copy(), e8.copy()
    if garbage:
        v8[:, :, :, fb:fb + nf], e8[:, :, :, fb:fb + nf] = 0x7f, 0xff
    values, exps = torch.from_numpy(v8).to(DEV), torch.from_numpy(e8).to(DEV)
    fresh = to_dev(ok.to_buffer(fk, fv), dtype) if nf else None
    out = torch.full((B, n_q, heads * d), float("nan"), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device=DEV)
    need = lib.attention_quantized_workspace_bytes(B, heads, n_q, N, d, code(dtype)) if split else 0
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device=DEV) if need else None
    lib.attention_quantized(to_dev(q, dtype), lib.quantized_kv(values, exps), fresh, 2 * nf * heads * d, fb, nf, B,
                            heads, n_q, d, out, code(dtype), workspace=ws)
    return to_host(out).reshape(B, n_q, heads, d).transpose(0, 2, 1, 3)


def check(got, dtype, q, K, V, tight=True):
    d, N = q.shape[-1], K.shape[2]
    ref, A = ok.attention(q, K, V, absolute=True)
    S = (np.abs(q) @ np.swapaxes(np.abs(K), -1, -2)).max(-1, keepdims=True) / np.sqrt(d)
    tol = A * (2.0 ** -22 * (d + 2) * S + 2.0 ** -20 + N * 2.0 ** -23)
    if dtype == "bf16":
        tol = tol + A * 2.0 ** -7 + np.abs(ref) * 2.0 ** -8
    worst = float((np.abs(got - ref) / tol).max())
    err = rel_l2(got, ref)
    print(f"  rel-L2 {err:.2e}, worst {worst:.3f} of the tolerance", flush=True)
    assert worst <= 1.0
    if tight:
        assert err <= NORM[dtype], err


SHAPES = [  # heads, n_q, n_kv, fresh_begin, n_fresh
    (1, 1, 1, 0, 0), (1, 1, 1, 0, 1), (3, 1, 200, 7, 1), (2, 2, 65, 64, 1), (2, 31, 64, 0, 64), (2, 33, 63, 5, 33),
    (4, 40, 128, 40, 40), (2, 65, 321, 100, 65), (2, 96, 256, 80, 96), (3, 130, 1000, 333, 130), (1, 300, 2025, 1035, 45),
    (2, 17, 4100, 0, 0), (16, 129, 640, 0, 640), (1, 1, 9000, 8990, 10), (8, 260, 1024, 512, 260),
    # short bands across chunks of eight keys and across tiles
    (2, 40, 200, 6, 5), (2, 9, 130, 60, 8), (1, 600, 130, 62, 7), (2, 70, 150, 61, 9), (1, 3, 70, 64, 6),
    # many queries: keys laid out as tiles once
    (2, 513, 1001, 333, 513), (1, 600, 640, 0, 640), (3, 512, 65, 3, 1), (1, 1100, 192, 64, 128), (2, 700, 1, 0, 0),
]


@pytest.mark.parametrize("split", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 72, 80, 96, 128])
@pytest.mark.parametrize("heads,n_q,N,fb,nf", SHAPES)
def test_attention(orch_lib, split, dtype, d, heads, n_q, N, fb, nf):
    print(f"\n[{dtype} d {d} heads {heads} n_q {n_q} n_kv {N} fresh {fb}+{nf} split {split}]", flush=True)
    rng = np.random.default_rng(d + n_q + N)
    q, v8, e8, fk, fv, K, V = make(rng, dtype, 2, heads, d, n_q, N, fb, nf)
    check(run(orch_lib, dtype, q, v8, e8, fk, fv, fb, split), dtype, q, K, V)


@pytest.mark.parametrize("split", [True, False])
@pytest.mark.parametrize("d", [32, 64, 72, 80, 96, 128])
@pytest.mark.parametrize("n_q,N,fb,nf", [(1100, 600, 77, 300), (1027, 333, 0, 0), (1100, 640, 64, 512), (520, 2000, 1001, 520)])
def test_many_heads_and_queries(orch_lib, split, d, n_q, N, fb, nf):
    """Enough workgroups that the keys are laid out as tiles once (with a workspace), or taken by whole workgroups."""
    print(f"\n[d {d} n_q {n_q} n_kv {N} fresh {fb}+{nf} split {split}]", flush=True)
    rng = np.random.default_rng(d + n_q + N)
    q, v8, e8, fk, fv, K, V = make(rng, "bf16", 2, 16, d, n_q, N, fb, nf)
    check(run(orch_lib, "bf16", q, v8, e8, fk, fv, fb, split), "bf16", q, K, V)


@pytest.mark.parametrize("d", [32, 64, 72, 80, 96, 128])
def test_keys_laid_out_and_split(orch_lib, d):
    """Tiles laid out once, and their keys over several workgroups."""
    n_q, N, fb, nf = 1500, 2025, 333, 900
    print(f"\n[d {d} n_q {n_q} n_kv {N} fresh {fb}+{nf}]", flush=True)
    rng = np.random.default_rng(d + n_q + N)
    q, v8, e8, fk, fv, K, V = make(rng, "bf16", 2, 6, d, n_q, N, fb, nf)
    check(run(orch_lib, "bf16", q, v8, e8, fk, fv, fb), "bf16", q, K, V)


@pytest.mark.parametrize("split", [True, False])
@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("ramp,shift", [(12.0, 0.0), (0.0, 48.0), (0.0, 2.0 ** 15)])
@pytest.mark.parametrize("dtype,B,heads,n_q,N", [("bf16", 1, 2, 70, 1000), ("bf16", 2, 16, 1100, 600), ("f32", 1, 2, 70, 1000)])
def test_running_max(orch_lib, split, dtype, d, ramp, shift, B, heads, n_q, N):
    """Scores that grow along the keys, and scores with a large common offset."""
    rng = np.random.default_rng(d)
    q, v8, e8, fk, fv, K, V = make(rng, dtype, B, heads, d, n_q, N, N // 2, 70, ramp, shift)
    print(f"\n[{dtype} d {d} ramp {ramp} shift {shift} split {split}]", flush=True)
    check(run(orch_lib, dtype, q, v8, e8, fk, fv, N // 2, split), dtype, q, K, V, tight=False)


# few queries (waves share the keys), whole workgroups, prepared tiles
SIZES = [(1, 2, 40, 200), (2, 16, 520, 330), (2, 16, 1100, 333)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("B,heads,n_q,N", SIZES)
def test_equal_huge_scores_are_a_mean(orch_lib, dtype, d, B, heads, n_q, N):
    """Every score the same number of 10^30 and more (either sign): the mean of V."""
    rng = np.random.default_rng(1)
    q, v8, e8, fk, fv, K, V = make(rng, dtype, B, heads, d, n_q, N, 0, 0)
    q[:], q[..., 0] = 0.0, 2.0 ** 60
    for sign in (1, -1):
        k = np.zeros_like(K)
        k[..., 0] = sign * 2.0 ** 50
        v8[:, 0], e8[:, 0] = ok.quantize(k)
        got = run(orch_lib, dtype, q, v8, e8, fk, fv, 0)
        check(got, dtype, np.zeros_like(q), k, V)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 72, 96])
@pytest.mark.parametrize("B,heads,n_q,N", SIZES)
def test_not_finite(orch_lib, dtype, d, B, heads, n_q, N):
    """A key whose score is minus infinity has no part in the result, wherever it lies; an infinite score or a NaN
    makes its own queries NaN and no others."""
    rng = np.random.default_rng(4)
    fb, nf = 60, 100
    q, v8, e8, fk, fv, K, V = make(rng, dtype, B, heads, d, n_q, N, fb, nf)
    q[..., 0] = np.abs(q[..., 0]) + 0.5
    out = []
    masked = [0, 1, 40, 99]
    for val in (-np.inf, np.inf, np.nan):
        f = fk.copy()
        f[:, 0, masked, 0] = val                       # head 0 only
        qq = q.copy()
        out.append(run(orch_lib, dtype, qq, v8, e8, f, fv, fb))
    keep = np.setdiff1d(np.arange(N), fb + np.array(masked))
    ref = ok.attention(q[:, :1], K[:, :1, keep], V[:, :1, keep])
    assert rel_l2(out[0][:, :1], ref) <= NORM[dtype]
    assert np.isnan(out[1][:, 0]).all() and np.isnan(out[2][:, 0]).all()
    for o in out:
        assert rel_l2(o[:, 1], ok.attention(q[:, 1], K[:, 1], V[:, 1])) <= NORM[dtype]
    # a NaN in the cache reaches every query of its head; one query's NaN itself alone
    v = v8.copy()
    v[0, 0, 1, 5, 3] = 0x7f
    got = run(orch_lib, dtype, q, v, e8, fk, fv, fb)
    assert np.isnan(got[0, 1]).all() and np.isfinite(got[0, 0]).all()
    qn = q.copy()
    qn[0, 0, 7, 2] = np.nan
    got = run(orch_lib, dtype, qn, v8, e8, fk, fv, fb)
    assert np.isnan(got[0, 0, 7]).all() and np.isfinite(np.delete(got[0, 0], 7, 0)).all()


@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("B,heads,n_q,N", SIZES)
def test_infinite_value(orch_lib, d, B, heads, n_q, N):
    """An infinite V of a fresh key: infinite in its channel, the others as they are."""
    rng = np.random.default_rng(6)
    q, v8, e8, fk, fv, K, V = make(rng, "bf16", B, heads, d, n_q, N, 10, 33)
    fv[0, 0, 20, 5] = np.inf
    got = run(orch_lib, "bf16", q, v8, e8, fk, fv, 10)[0, 0]
    V[0, 0, 30, 5] = 0.0
    assert np.isinf(got[..., 5]).all()
    c = np.arange(d) != 5
    assert rel_l2(got[..., c], ok.attention(q[0, 0], K[0, 0], V[0, 0])[..., c]) <= NORM["bf16"]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_agrees_with_attention_over_the_read_back_buffer(orch_lib, dtype):
    """The same result as reading the cache back and calling the attention of the operand type."""
    B, heads, d, n_q, N, fb = 2, 4, 72, 128, 512, 128
    rng = np.random.default_rng(8)
    q, v8, e8, fk, fv, K, V = make(rng, dtype, B, heads, d, n_q, N, fb, n_q)
    got = run(orch_lib, dtype, q, v8, e8, fk, fv, fb, garbage=False)
    H = heads * d
    values, exps = torch.from_numpy(v8).to(DEV), torch.from_numpy(e8).to(DEV)
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    stale, out = torch.empty((B, 2 * N * H), dtype=td, device=DEV), torch.empty((B, n_q, H), dtype=td, device=DEV)
    orch_lib.kv_dequantize(orch_lib.quantized_kv(values, exps), 0, stale, 2 * N * H, N, 0, B, heads, N, d, code(dtype))
    orch_lib.attention(to_dev(q, dtype), stale, 2 * N * H, to_dev(ok.to_buffer(fk, fv), dtype), 2 * n_q * H, fb, n_q, B,
                       heads, n_q, N, d, out, code(dtype))
    ref = to_host(out).reshape(B, n_q, heads, d).transpose(0, 2, 1, 3)
    assert rel_l2(got, ref) <= 2 * NORM[dtype]


@pytest.mark.parametrize("dtype,n_q", [("bf16", 1), ("bf16", 300), ("f32", 1)])
def test_a_long_cache(orch_lib, dtype, n_q):
    """More than 2^32 bytes from the first value to the last; all but a few keys, at both ends of it and between, at
    scores 224 below 0, whose probabilities are 0 in fp32."""
    heads, d, N, nf = 2, 64, 2 ** 24 + 70, 33
    fb, at = N - 50, np.array([0, 1, 2 ** 23 + 5, 2 ** 24 - 1, N - 1])
    values = torch.zeros((1, 2, heads, N, d), dtype=torch.uint8, device=DEV)
    exps = torch.full((1, 2, heads, N), 127, dtype=torch.uint8, device=DEV)
    assert values.numel() > 2 ** 32
    values[:, 0, :, :, 0] = 0xfe                       # -448
    values[:, 1] = 0x40                                # 2
    q, v8, e8, fk, fv, K, V = make(np.random.default_rng(13), dtype, 1, heads, d, n_q, len(at) + nf, len(at), nf)
    q[..., 0], K[..., 0], fk[..., 0] = 4.0, 0.0, 0.0
    v8[:, 0, :, :, 0] = 0
    for i, n in enumerate(at):
        values[:, :, :, n], exps[:, :, :, n] = torch.from_numpy(v8[:, :, :, i]).to(DEV), torch.from_numpy(e8[:, :, :, i]).to(DEV)
    cache = orch_lib.quantized_kv(values, exps)
    fresh = to_dev(ok.to_buffer(fk, fv), dtype)
    need = orch_lib.attention_quantized_workspace_bytes(1, heads, n_q, N, d, code(dtype))
    for ws in (None, torch.empty(need, dtype=torch.uint8, device=DEV)):
        out = torch.empty((1, n_q, heads * d), dtype=fresh.dtype, device=DEV)
        orch_lib.attention_quantized(to_dev(q, dtype), cache, fresh, 0, fb, nf, 1, heads, n_q, d, out, code(dtype), workspace=ws)
        check(to_host(out).reshape(1, n_q, heads, d).transpose(0, 2, 1, 3), dtype, q, K, V)


def test_rows_and_neighbours_untouched(orch_lib):
    """No query, and what lies behind the output."""
    rng = np.random.default_rng(9)
    q, v8, e8, fk, fv, K, V = make(rng, "bf16", 1, 2, 72, 37, 100, 0, 0)
    values, exps = torch.from_numpy(v8).to(DEV), torch.from_numpy(e8).to(DEV)
    cache = orch_lib.quantized_kv(values, exps)
    out = torch.full((37 * 144 + 512,), 7.0, dtype=torch.bfloat16, device=DEV)
    orch_lib.attention_quantized(to_dev(q, "bf16"), cache, None, 0, 0, 0, 1, 2, 0, 72, out, 1)
    torch.cuda.synchronize()
    assert torch.all(out == 7)
    orch_lib.attention_quantized(to_dev(q, "bf16"), cache, None, 0, 0, 0, 1, 2, 37, 72, out, 1)
    torch.cuda.synchronize()
    assert torch.all(out[37 * 144:] == 7) and not torch.any(out[:37 * 144] == 7)


@pytest.mark.parametrize("dtype,B,heads,d,n_q,N", [("bf16", 2, 16, 72, 1100, 600), ("bf16", 1, 2, 64, 20, 5000), ("f32", 1, 2, 64, 20, 5000)])
def test_a_workspace_is_used_whole_or_not_at_all(orch_lib, dtype, B, heads, d, n_q, N):
    """Fewer bytes than asked for: the bits of a call without one, and nothing written past the bytes that are there."""
    rng = np.random.default_rng(11)
    q, v8, e8, fk, fv, K, V = make(rng, dtype, B, heads, d, n_q, N, 0, 0)
    qd, values, exps = to_dev(q, dtype), torch.from_numpy(v8).to(DEV), torch.from_numpy(e8).to(DEV)
    cache = orch_lib.quantized_kv(values, exps)
    need = orch_lib.attention_quantized_workspace_bytes(B, heads, n_q, N, d, code(dtype))
    assert need > 0
    ws = torch.full((need + 256,), 0x5a, dtype=torch.uint8, device=DEV)
    outs = []
    for bytes_ in (None, 16, need - 1, need):
        out = torch.empty((B, n_q, heads * d), dtype=qd.dtype, device=DEV)
        orch_lib.attention_quantized(qd, cache, None, 0, 0, 0, B, heads, n_q, d, out, code(dtype),
                                     workspace=None if bytes_ is None else ws[:bytes_])
        outs.append(out)
        if bytes_ != need:
            assert torch.all(ws == 0x5a)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    assert torch.all(ws[need:] == 0x5a) and not torch.all(ws[:need] == 0x5a)
    for out in (outs[0], outs[3]):
        check(to_host(out).reshape(B, n_q, heads, d).transpose(0, 2, 1, 3), dtype, q, K, V)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [72, 128])
def test_repeated_calls_give_the_same_bits(orch_lib, dtype, d):
    """No order of waves or workgroups shows: ten calls of each variant, bit for bit."""
    for B, heads, n_q, N, fb, nf in ((1, 2, 40, 330, 50, 40), (2, 16, 520, 333, 0, 0), (2, 16, 1100, 640, 64, 512)):
        rng = np.random.default_rng(12)
        q, v8, e8, fk, fv, K, V = make(rng, dtype, B, heads, d, n_q, N, fb, nf)
        first = run(orch_lib, dtype, q, v8, e8, fk, fv, fb)
        for _ in range(9):
            np.testing.assert_array_equal(run(orch_lib, dtype, q, v8, e8, fk, fv, fb), first)


@pytest.mark.parametrize("d", [32, 64, 72, 80, 96, 128])
@pytest.mark.parametrize("B,heads,n_q,N,fb,nf", [(2, 8, 96, 256, 80, 96), (2, 8, 45, 2025, 1035, 45), (2, 16, 520, 330, 60, 100),
                                                 (2, 16, 1100, 600, 77, 300)])
def test_error_is_the_rounding_of_the_output(orch_lib, d, B, heads, n_q, N, fb, nf):
    """bf16: probabilities reach the products with 16 bits (off by 2^-17), so that the output's own rounding is what is
    left.  Half a step of 2^-7 of a value's power of two is evenly spread: 2^-8 / sqrt(3) over the value's mantissa,
    0.736 of it in the 2-norm over evenly spread exponents, 1.66e-3, 1.70e-3 at most for normal outputs of any size
    (probabilities rounded to bf16 once add as much again: 2.35e-3).  24000 outputs and more: 2% either way."""
    rng = np.random.default_rng(d + n_q + N)
    q, v8, e8, fk, fv, K, V = make(rng, "bf16", B, heads, d, n_q, N, fb, nf)
    for split in (True, False):
        err = rel_l2(run(orch_lib, "bf16", q, v8, e8, fk, fv, fb, split), ok.attention(q, K, V))
        print(f"\n[d {d} {heads} heads, {n_q} queries x {N} keys, split {split}] {err:.3e}", flush=True)
        assert err <= 1.75e-3


@pytest.mark.parametrize("n_q,groups", [(2, 1), (1000, 4)])
def test_a_long_band(orch_lib, n_q, groups):
    """A band of nearly 2^31 channels a head, its rows of V^T more than 2^31 bytes apart within a workgroup's reach; all but a
    few keys at scores 224 below 0, whose probabilities are 0 in fp32."""
    d, N = 32, 2 ** 26 - 64
    at = np.array([0, 1, 77, 2 ** 25 + 5, 2 ** 26 - 200, N - 1])
    values = torch.full((1, 2, 1, N, d), 0x7f, dtype=torch.uint8, device=DEV)           # not to be read
    exps = torch.full((1, 2, 1, N), 127, dtype=torch.uint8, device=DEV)
    fresh = torch.zeros(2 * N * d, dtype=torch.bfloat16, device=DEV)
    k, vt = fresh[:N * d].view(N, d), fresh[N * d:].view(d, N)
    k[:, 0] = -448.0 * 2 ** 0.5 / 2                                                     # times 4 / sqrt(32): -224
    vt[:] = 2.0
    q, _, _, fk, fv, K, V = make(np.random.default_rng(14), "bf16", 1, 1, d, n_q, len(at), 0, len(at))
    q[..., 0], K[..., 0], fk[..., 0] = 4.0, 0.0, 0.0
    for i, n in enumerate(at):
        k[n], vt[:, n] = to_dev(fk[0, 0, i], "bf16"), to_dev(fv[0, 0, i], "bf16")
    cache = orch_lib.quantized_kv(values, exps)
    need = orch_lib.attention_quantized_workspace_bytes(1, 1, n_q, N, d, 1)
    assert orch_lib.attention_quantized_plan(1, 1, n_q, N, d, 1, need)[1] == groups
    for ws in (None, torch.empty(need, dtype=torch.uint8, device=DEV)):
        out = torch.empty((1, n_q, d), dtype=torch.bfloat16, device=DEV)
        orch_lib.attention_quantized(to_dev(q, "bf16"), cache, fresh, 0, 0, N, 1, 1, n_q, d, out, 1, workspace=ws)
        check(to_host(out).reshape(1, n_q, 1, d).transpose(0, 2, 1, 3), "bf16", q, K, V)
