"""Norms of rows as large as the header allows: their sum of squares (about the mean for a LayerNorm) just below
the largest fp32, 2^128."""
import numpy as np
import pytest

from tests.test_gpu_block_norms import _run

pytestmark = pytest.mark.gpu


def _rows(rng, rows, H):
    """Deviations around 0 whose squares sum to 0.95 * 2^128: 0.974 * 2^64 / sqrt(H) in the root mean square
    (their sum of H values stays below 2^64 sqrt(H), and H + 50 roundings of 2^-24 below the 5% left)."""
    x = rng.standard_normal((rows, H))
    x -= x.mean(1, keepdims=True)
    return x * (np.sqrt(0.95) * 2.0 ** 64 / np.sqrt((x * x).sum(1, keepdims=True)))


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("H", [4, 61, 1152, 2304, 12000, 32768])
@pytest.mark.parametrize("codes", [False, True])
def test_largest_stream(orch_lib, kind, H, codes):
    rng = np.random.default_rng(H)
    _run(orch_lib, rng, 5, H, "f32", pre=kind, affine=False, mod=False, y=False, codes=codes, h=_rows(rng, 5, H))


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("H", [61, 1152, 12000])
def test_largest_output_of_a_block(orch_lib, kind, H):
    rng = np.random.default_rng(H)
    _run(orch_lib, rng, 5, H, "f32", post=kind, affine=False, mod=False, yv=_rows(rng, 5, H).astype(np.float32).astype(np.float64))
