"""The norms around a block and the 8-bit integer products at sizes past 32 bits of one kind or another."""
import numpy as np
import pytest
import torch

from oracle import integer as oi
from tests._gpu_util import DEV, to_host

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def test_wide_rows_past_a_grid(orch_lib):
    """2^22 rows and more of a workgroup of 1024 threads each: more threads than 32 bits count.  In place,
    so that a row that is taken twice or not at all shows."""
    lib = orch_lib
    rows, H = (1 << 22) + 3, 5124                        # 86 GB
    free, _ = torch.cuda.mem_get_info()
    if free < 100 << 30:
        pytest.skip("needs 100 GiB of free device memory")
    h = torch.ones((rows, H), device=DEV)
    some = [0, 1, (1 << 21) - 1, 1 << 21, (1 << 21) + 1, (1 << 22) - 1, 1 << 22, rows - 1]
    x = np.random.default_rng(0).standard_normal((len(some), H)).astype(np.float32)
    for i, r in enumerate(some):
        h[r] = torch.from_numpy(x[i]).to(DEV)
    lib.block_norms(h, None, h, residual_scale=0.5)
    torch.cuda.synchronize()
    for i, r in enumerate(some):
        np.testing.assert_array_equal(h[r].cpu().numpy(), 0.5 * x[i])
        h[r] = 0.5
    for part in h.split(1 << 18):
        lo, hi = torch.aminmax(part)
        assert float(lo) == 0.5 and float(hi) == 0.5
    del h, part
    torch.cuda.empty_cache()
