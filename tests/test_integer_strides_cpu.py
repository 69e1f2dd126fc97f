"""Strides whose rows reach past 64-bit addresses are refused (checked before anything is launched, so no
GPU is needed; the pointers are never read)."""
import ctypes as C

import pytest

F32, BF16 = 0, 1
P = [0x10000000 * (i + 1) for i in range(16)]      # addresses far apart, 16-byte aligned
ROWS = (1 << 23) + 1                               # 2^23 strides of 2^39 fp32 elements: 2^64 bytes


def _refused(lib, rc):
    assert rc == lib.ORCH_EINVAL and "address" in lib.last_error(), (rc, lib.last_error())


@pytest.mark.parametrize("dtype,stride", [(F32, 1 << 39), (BF16, (1 << 40) - 1)])
@pytest.mark.parametrize("name", ["h_stride", "y_stride", "h_out_stride", "out_stride", "mod_stride"])
def test_norms(orch_lib, name, dtype, stride):
    lib = orch_lib
    p = lib.BlockNorms()
    for i, k in enumerate(("h", "y", "gate", "shift", "scale", "h_out", "out")):
        setattr(p, k, P[i])
    p.rows, p.hidden, p.rows_per_batch, p.residual_scale = ROWS, 32, 1, 1.0
    for k in ("h_stride", "y_stride", "h_out_stride", "out_stride", "mod_stride"):
        setattr(p, k, 32)
    setattr(p, name, stride)
    _refused(lib, lib.lib.orch_op_block_norms(C.byref(p), dtype, None))


def test_norms_hidden_by_a_wrap(orch_lib):
    """2^23 strides of 2^41 bytes come to 2^64: taken as one row, h would not overlap h_out behind it."""
    lib = orch_lib
    p = lib.BlockNorms()
    p.rows, p.hidden, p.residual_scale, p.h, p.h_out = ROWS, 32, 1.0, P[0], P[0] + 4096
    p.h_stride, p.h_out_stride = 1 << 39, 32
    _refused(lib, lib.lib.orch_op_block_norms(C.byref(p), BF16, None))


@pytest.mark.parametrize("dtype,stride", [(F32, 1 << 39), (BF16, (1 << 40) - 1)])
def test_quantize(orch_lib, dtype, stride):
    lib = orch_lib
    out = lib.Int8Rows(P[1], P[2], 48)
    _refused(lib, lib.lib.orch_op_quantize_rows(P[0], stride, ROWS, 40, C.byref(out), dtype, None))


def _operands(lib):
    return C.byref(lib.Int8Rows(P[0], P[1], 48)), C.byref(lib.Int8Rows(P[2] << 8, P[3], 48))


@pytest.mark.parametrize("stride", [1 << 39, (1 << 40) - 1])
def test_gate(orch_lib, stride):
    A, W = _operands(orch_lib)
    rc = orch_lib.lib.orch_op_linear_quantized(A, ROWS, 40, W, 24, None, 2, P[5] << 8, stride, 1, P[6] << 8, None, 0, F32, None)
    _refused(orch_lib, rc)


@pytest.mark.parametrize("dtype,stride", [(F32, 1 << 39), (BF16, (1 << 40) - 8)])
def test_kv_branches(orch_lib, dtype, stride):
    A, W = _operands(orch_lib)
    rc = orch_lib.lib.orch_op_qkv_projection_quantized(A, ROWS, 1, 40, W, None, 1, 32, P[6] << 8, P[7] << 8, stride, 4, 0, None, 0,
                                                       dtype, None)
    _refused(orch_lib, rc)
