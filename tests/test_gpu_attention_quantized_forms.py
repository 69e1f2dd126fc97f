"""Every form of the attention over the 8-bit cache at every head size, by shapes for which the library says that it runs in
that form: against the float64 oracle, with keys that take no part, infinities and large scores, bit for bit again.
Tolerances as in test_gpu_attention_quantized.py."""
import numpy as np
import pytest

from oracle import kvcache as ok
from tests._attention_forms import FORMS, SIZES, shape_for
from tests._gpu_util import rel_l2
from tests.test_gpu_attention_quantized import NORM, check, make, run

pytestmark = pytest.mark.gpu

CASES = [(form, d) for form in FORMS for d in SIZES]
IDS = ["-".join([f[0], "prepared" if f[1] else f"groups{f[2]}", "split" if f[3] else "whole", str(d)]) for f, d in CASES]


def _inputs(lib, form, d):
    B, heads, n_q, N, ws = shape_for(lib, form, d)
    fb = N // 3 | 1
    nf = min(n_q, N - fb - 2)
    print(f"\n[{form} d {d}: {B} x {heads} heads, {n_q} queries x {N} keys, fresh {fb}+{nf}]", flush=True)
    return make(np.random.default_rng(d + N), form[0], B, heads, d, n_q, N, fb, nf), fb, nf, N, ws


@pytest.mark.parametrize("form,d", CASES, ids=IDS)
def test_against_the_oracle(orch_lib, form, d):
    (q, v8, e8, fk, fv, K, V), fb, _, _, ws = _inputs(orch_lib, form, d)
    first = run(orch_lib, form[0], q, v8, e8, fk, fv, fb, ws)
    check(first, form[0], q, K, V)
    for _ in range(4):
        np.testing.assert_array_equal(run(orch_lib, form[0], q, v8, e8, fk, fv, fb, ws), first)


@pytest.mark.parametrize("form,d", CASES, ids=IDS)
def test_keys_without_a_part(orch_lib, form, d):
    """Scores of minus infinity at both ends of the band and across a tile's edge, and a head whose
    every fresh key is one: the attention of the other keys."""
    (q, v8, e8, fk, fv, K, V), fb, nf, N, ws = _inputs(orch_lib, form, d)
    q[..., 0] = np.abs(q[..., 0]) + 0.5
    masked = np.unique(np.clip([0, nf // 2, nf - 1, 64 - fb % 64], 0, nf - 1))
    fk[:, 0, masked, 0] = -np.inf
    fk[:, -1, :, 0] = -np.inf
    got = run(orch_lib, form[0], q, v8, e8, fk, fv, fb, ws)
    for h, out in ((0, masked), (q.shape[1] - 1, np.arange(nf))):
        keep = np.setdiff1d(np.arange(N), fb + out)
        assert rel_l2(got[:, h], ok.attention(q[:, h], K[:, h, keep], V[:, h, keep])) <= NORM[form[0]]


@pytest.mark.parametrize("form,d", CASES, ids=IDS)
def test_large_equal_scores_and_infinite_values(orch_lib, form, d):
    """Scores of 10^30 and more, all the same: the mean of V.  An infinite V of a fresh key: infinite in its channel."""
    (q, v8, e8, fk, fv, K, V), fb, nf, N, ws = _inputs(orch_lib, form, d)
    at, c = (0, 0, nf // 2, 5), np.arange(d) != 5
    f = fv.copy()
    f[at] = np.inf
    got = run(orch_lib, form[0], q, v8, e8, fk, f, fb, ws)
    assert np.isinf(got[0, 0, :, 5]).all()
    assert rel_l2(got[0, 0][:, c], ok.attention(q[0, 0], K[0, 0], V[0, 0])[:, c]) <= NORM[form[0]]
    q[:], q[..., 0] = 0.0, 2.0 ** 60
    for sign in (1, -1):
        k = np.zeros_like(K)
        k[..., 0] = sign * 2.0 ** 50
        v8[:, 0], e8[:, 0] = ok.quantize(k)
        check(run(orch_lib, form[0], q, v8, e8, k[:, :, fb:fb + nf], fv, fb, ws), form[0], np.zeros_like(q), k, V)
