"""Sizes that the 8-bit integer operators' C arguments do not hold, refused by the binding (tensors
without memory; nothing is launched)."""
import pytest
import torch

BIG = 1 << 32          # an int's bits of it: 0


def _rows(lib, rows, cols):
    return lib.int8_rows(torch.empty((rows, cols), dtype=torch.int8, device="meta"), torch.empty(rows, device="meta"))


@pytest.fixture
def lib(orch_lib, monkeypatch):
    """The binding up to its call, as if the tensors were on the current GPU."""
    monkeypatch.setattr(orch_lib, "_stream_here", lambda *a: None)
    return orch_lib


def _raises(lib, f):
    with pytest.raises(lib.OrchError) as e:
        f()
    assert e.value.code == lib.ORCH_EINVAL and "int's range" in str(e.value), str(e.value)


@pytest.mark.parametrize("rows,cols", [(BIG, 64), (BIG + 5, 64), (1 << 31, 1), (0, BIG), (0, BIG + 64)])
def test_rows_past_an_int(lib, rows, cols):
    x = torch.empty((rows, cols), device="meta")
    _raises(lib, lambda: lib.quantize_rows(x, _rows(lib, rows, cols)))


@pytest.mark.parametrize("M,K,N", [(BIG, 64, 96), (0, BIG + 64, 96), (0, 64, BIG + 96), (0, 64, 1 << 31)])
def test_products_past_an_int(lib, M, K, N):
    out = torch.empty((M, N), device="meta")
    _raises(lib, lambda: lib.linear_quantized(_rows(lib, M, K), _rows(lib, N, K), None, lib.EPI_STORE, out))


@pytest.mark.parametrize("B,n,K,N", [(1, BIG, 64, 96), (2, BIG, 64, 96), (1, 0, BIG + 64, 96), (BIG + 1, 0, 64, 96), (1, 0, 64, 3 * (BIG + 32))])
def test_qkv_past_an_int(lib, B, n, K, N):
    q, kv = torch.empty((B, 1, n, N // 3), device="meta"), torch.empty((B, 2 * 8 * N // 3), device="meta")
    _raises(lib, lambda: lib.qkv_projection_quantized(_rows(lib, B * n, K), _rows(lib, N, K), None, q, kv, 8, 0))


@pytest.mark.parametrize("epilogue", [BIG, -BIG, BIG + 1])
def test_epilogue_past_an_int(lib, epilogue):
    _raises(lib, lambda: lib.linear_quantized(_rows(lib, 0, 64), _rows(lib, 96, 64), None, epilogue, torch.empty((0, 96), device="meta")))


@pytest.mark.parametrize("rows,hidden", [(1 << 31, 1), (BIG, 64), (0, 1 << 31), (0, BIG + 64)])
def test_norms_past_an_int(lib, rows, hidden):
    h = torch.empty((rows, hidden), device="meta")
    _raises(lib, lambda: lib.block_norms(h, None, h))


@pytest.mark.parametrize("scale", [1e39, -1e39, float("inf"), float("nan")])
def test_residual_scale_past_fp32(lib, scale):
    h = torch.empty((4, 32), device="meta")
    with pytest.raises(lib.OrchError) as e:
        lib.block_norms(h, None, h, residual_scale=scale)
    assert e.value.code == lib.ORCH_EINVAL and "residual_scale" in str(e.value), str(e.value)
