"""ctypes binding of liborch.so (argument marshalling only).

Every function here forwards to the C ABI declared in include/orch.h; all
computation happens in the library's HIP kernels.  PyTorch is used only to
hold device memory and to name the current HIP stream.  Importing this
module raises if the library has not been built.
"""
from __future__ import annotations

import ctypes as C
import os
import struct

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "liborch.so")

ORCH_OK, ORCH_EINVAL, ORCH_ENOWEIGHTS, ORCH_EHIP, ORCH_ENOMEM = 0, -1, -2, -3, -4
ORCH_F32, ORCH_BF16 = 0, 1
EPI_STORE, EPI_GELU, EPI_RESIDUAL = 0, 1, 2
DTYPE_CODE = {"f32": ORCH_F32, "bf16": ORCH_BF16}
NORM_CODE = {"none": 0, "layer": 1, "rms": 2}

SYMBOLS = (
    "orch_create", "orch_destroy", "orch_load_dit_weights", "orch_stale_kv_bytes",
    "orch_patch_denoise_step", "orch_scheduler_update", "orch_schedule_coefficients",
    "orch_last_error", "orch_op_layernorm_modulate", "orch_op_linear", "orch_op_qkv_projection",
    "orch_op_attention", "orch_op_conditioning", "orch_op_patch_embed", "orch_op_final_layer",
    "orch_attention_workspace_bytes", "orch_set_kernel_timing", "orch_kernel_times",
    "orch_linear_workspace_bytes",
    "orch_plan_devices", "orch_sample_patch_parallel", "orch_set_work_split",
    "orch_op_attention_noalloc", "orch_speeds_from_profiles", "orch_unet_conv_band",
    "orch_unet_conv_workspace_bytes", "orch_op_rotary", "orch_op_kv_quantize",
    "orch_op_kv_dequantize", "orch_op_attention_quantized",
    "orch_attention_quantized_workspace_bytes", "orch_attention_quantized_plan",
    "orch_op_block_norms", "orch_op_quantize_rows", "orch_op_linear_quantized",
    "orch_linear_quantized_workspace_bytes", "orch_op_qkv_projection_quantized",
)
KCLASSES = ("conditioning", "patch_embed", "layernorm", "qkv_gemm", "attention", "proj_gemm",
            "fc1_gemm", "fc2_gemm", "final_layer", "update")


class OrchError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"orch error {code}: {msg}")
        self.code = code


class UNetConvShape(C.Structure):
    _fields_ = [("height", C.c_int), ("width", C.c_int), ("channels", C.c_int),
                ("groups", C.c_int), ("out_channels", C.c_int), ("eps", C.c_float)]


class RotaryAxes(C.Structure):
    _fields_ = [("channels", C.c_int * 3), ("extent", C.c_int * 3), ("origin", C.c_double * 3),
                ("step", C.c_double * 3), ("theta", C.c_double), ("interleaved", C.c_int)]


class RotaryTensor(C.Structure):
    _fields_ = [("x", C.c_void_p), ("out", C.c_void_p), ("heads", C.c_int),
                ("x_stride", C.c_size_t * 3), ("out_stride", C.c_size_t * 3)]


class QuantizedKV(C.Structure):
    _fields_ = [("values", C.c_void_p), ("exponents", C.c_void_p), ("values_stride", C.c_size_t),
                ("exponents_stride", C.c_size_t), ("tokens", C.c_int)]


class Int8Rows(C.Structure):
    _fields_ = [("values", C.c_void_p), ("scales", C.c_void_p), ("stride", C.c_size_t)]


class Norm(C.Structure):
    _fields_ = [("kind", C.c_int), ("eps", C.c_float), ("weight", C.c_void_p), ("bias", C.c_void_p)]


class BlockNorms(C.Structure):
    _fields_ = [("post", Norm), ("pre", Norm), ("residual_scale", C.c_float), ("rows", C.c_int),
                ("hidden", C.c_int), ("rows_per_batch", C.c_int), ("h", C.c_void_p), ("y", C.c_void_p),
                ("gate", C.c_void_p), ("shift", C.c_void_p), ("scale", C.c_void_p), ("h_out", C.c_void_p),
                ("out", C.c_void_p), ("out8", C.POINTER(Int8Rows)), ("h_stride", C.c_size_t),
                ("y_stride", C.c_size_t), ("mod_stride", C.c_size_t), ("h_out_stride", C.c_size_t),
                ("out_stride", C.c_size_t)]


class OrchConfig(C.Structure):
    _fields_ = [("n_blocks", C.c_int), ("hidden", C.c_int), ("heads", C.c_int),
                ("mlp_hidden", C.c_int), ("in_ch", C.c_int), ("out_ch", C.c_int),
                ("patch", C.c_int), ("latent", C.c_int), ("num_classes", C.c_int),
                ("freq_dim", C.c_int), ("cfg_batch", C.c_int), ("dtype", C.c_int),
                ("T", C.c_int), ("beta_start", C.c_double), ("beta_end", C.c_double)]


def config_from(cfg) -> OrchConfig:
    """Build the C config from any object with the DiT shape attributes."""
    return OrchConfig(cfg.n_blocks, cfg.hidden, cfg.heads, cfg.mlp_hidden, cfg.in_ch, cfg.out_ch,
                      cfg.patch, cfg.latent, cfg.num_classes, cfg.freq_dim, cfg.cfg_batch,
                      DTYPE_CODE[cfg.dtype], cfg.T, cfg.beta_start, cfg.beta_end)


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with "
                          "`python -m paper_2509_04719_amd.build`")
    lib = C.CDLL(LIB_PATH)
    vp, i, sz, d, f = C.c_void_p, C.c_int, C.c_size_t, C.c_double, C.c_float
    sig = {
        "orch_create": (i, [C.POINTER(OrchConfig), C.POINTER(vp)]),
        "orch_destroy": (None, [vp]),
        "orch_load_dit_weights": (i, [vp, vp, sz]),
        "orch_stale_kv_bytes": (sz, [vp]),
        "orch_patch_denoise_step": (i, [vp, vp, i, i, i, i, C.POINTER(i), f, vp, i, vp, f, vp, vp,
                                        vp]),
        "orch_scheduler_update": (i, [vp, vp, vp, f, vp, d, d, d, vp, sz, vp]),
        "orch_schedule_coefficients": (i, [C.POINTER(OrchConfig), i, i, d, C.POINTER(d)]),
        "orch_last_error": (C.c_char_p, []),
        "orch_op_layernorm_modulate": (i, [vp, i, i, i, vp, vp, i, vp, i, vp]),
        "orch_op_linear": (i, [vp, i, i, vp, i, vp, i, vp, i, i, vp, vp, sz, i, vp]),
        "orch_linear_workspace_bytes": (sz, [i, i, i, i]),
        "orch_op_qkv_projection": (i, [vp, i, i, i, vp, vp, i, i, vp, vp, sz, i, i, i, vp]),
        "orch_op_attention": (i, [vp, vp, sz, vp, sz, i, i, i, i, i, i, i, vp, vp, sz, i, vp]),
        "orch_attention_workspace_bytes": (sz, [i, i, i, i, i, i]),
        "orch_op_attention_noalloc": (i, [vp, vp, sz, vp, sz, i, i, i, i, i, i, i, vp, i, vp]),
        "orch_set_kernel_timing": (i, [vp, i]),
        "orch_set_work_split": (i, [vp, i]),
        "orch_kernel_times": (i, [vp, C.POINTER(d), C.POINTER(C.c_longlong)]),
        "orch_op_conditioning": (i, [vp, i, C.POINTER(i), vp, vp]),
        "orch_op_patch_embed": (i, [vp, vp, i, i, vp, vp]),
        "orch_op_final_layer": (i, [vp, vp, i, i, vp, vp, vp]),
        "orch_plan_devices": (i, [C.POINTER(d), i, i, i, d, d, i, C.POINTER(i), C.POINTER(i)]),
        "orch_speeds_from_profiles": (i, [i, C.POINTER(i), C.POINTER(i), C.POINTER(d), i,
                                          C.POINTER(d)]),
        "orch_unet_conv_workspace_bytes": (sz, [C.POINTER(UNetConvShape), i]),
        "orch_unet_conv_band": (i, [C.POINTER(UNetConvShape), i, i, vp, vp, vp, vp, vp, vp, vp, i,
                                    vp, vp, sz, vp]),
        "orch_op_rotary": (i, [C.POINTER(RotaryAxes), vp, i, i, i, i, i, i, vp]),
        "orch_op_kv_quantize": (i, [vp, sz, i, i, C.POINTER(QuantizedKV), i, i, i, i, i, i, vp]),
        "orch_op_kv_dequantize": (i, [C.POINTER(QuantizedKV), i, vp, sz, i, i, i, i, i, i, i, vp]),
        "orch_op_attention_quantized": (i, [vp, C.POINTER(QuantizedKV), vp, sz, i, i, i, i, i, i, vp,
                                            vp, sz, i, vp]),
        "orch_attention_quantized_workspace_bytes": (sz, [i, i, i, i, i, i]),
        "orch_attention_quantized_plan": (i, [i, i, i, i, i, i, sz] + [C.POINTER(i)] * 3),
        "orch_op_block_norms": (i, [vp, i, vp]),
        "orch_op_quantize_rows": (i, [vp, sz, i, i, C.POINTER(Int8Rows), i, vp]),
        "orch_op_linear_quantized": (i, [C.POINTER(Int8Rows), i, i, C.POINTER(Int8Rows), i, vp, i, vp, sz, i, vp, vp, sz, i, vp]),
        "orch_linear_quantized_workspace_bytes": (sz, [i, i, i]),
        "orch_op_qkv_projection_quantized": (i, [C.POINTER(Int8Rows), i, i, i, C.POINTER(Int8Rows), vp, i, i, vp, vp, sz, i, i,
                                            vp, sz, i, vp]),
        "orch_sample_patch_parallel": (i, [vp, vp, i, C.POINTER(i), C.POINTER(i), C.POINTER(i), i, i,
                                           C.POINTER(i), f, vp, vp, vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


lib = _load()


def last_error() -> str:
    return lib.orch_last_error().decode()


def check(rc: int) -> None:
    if rc != ORCH_OK:
        raise OrchError(rc, last_error())


def _ptr(t):
    """Device address of a torch tensor (or None), as the pointer arguments take it."""
    return None if t is None else t.data_ptr()


def _stream(stream=None):
    """The handle of a torch stream, of the current one by default (straight from torch's
    runtime: a Stream object costs 3 us a call)."""
    import torch
    if stream is not None:
        return stream.cuda_stream
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _stream_on(stream, *devices):
    """The stream's handle, for tensors (their Tensor.get_device(), -1 on the host) that all have to
    be on the current GPU."""
    import torch
    cur = torch.cuda.current_device()
    for d in devices:
        if d != cur:
            raise OrchError(ORCH_EINVAL, f"a tensor is on {'the host' if d < 0 else f'GPU {d}'}, the current GPU is {cur}")
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(cur)
    if stream.device_index != cur:
        raise OrchError(ORCH_EINVAL, f"the stream is on GPU {stream.device_index}, the current GPU is {cur}")
    return stream.cuda_stream


def _check_ints(*values):
    """What a C int holds: ctypes wraps the rest silently."""
    if max(values) > 0x7fffffff or min(values) < -0x80000000:
        raise OrchError(ORCH_EINVAL, f"{values}: past an int's range")


_F32 = None


def _f32():
    """torch.float32 (torch is not imported before the first use)."""
    global _F32
    if _F32 is None:
        import torch
        _F32 = torch.float32
    return _F32


_CODES = {}             # by torch type, filled at the first use (torch is not imported before)


def _code(t):
    """The library's code of a tensor's type."""
    code = _CODES.get(t.dtype)
    if code is None:
        import torch
        _CODES.update({torch.float32: ORCH_F32, torch.bfloat16: ORCH_BF16})
        code = _CODES.get(t.dtype)
        if code is None:
            raise OrchError(ORCH_EINVAL, f"type {t.dtype} not supported")
    return code


def schedule_coefficients(cfg, t: int, t_prev: int, eta: float = 0.0):
    """(a, b, c) of x_prev = a x - b eps + c z, computed by the library (host)."""
    out = (C.c_double * 3)()
    oc = config_from(cfg)
    check(lib.orch_schedule_coefficients(C.byref(oc), t, t_prev, eta, out))
    return out[0], out[1], out[2]


def plan_devices(speeds, m_base, m_warmup, a, b, total_rows):
    """(steps, rows) per device from the library's planner (host only)."""
    n = len(speeds)
    v = (C.c_double * n)(*[float(x) for x in speeds])
    st = (C.c_int * n)()
    rw = (C.c_int * n)()
    check(lib.orch_plan_devices(v, n, m_base, m_warmup, float(a), float(b), total_rows, st, rw))
    return list(st), list(rw)


def speeds_from_profiles(profiles, ref_rows):
    """Effective speeds from per-device [(rows, ms), ...] profiles (host only)."""
    n = len(profiles)
    pts = [pt for prof in profiles for pt in prof]
    npts = (C.c_int * n)(*[len(prof) for prof in profiles])
    rows = (C.c_int * len(pts))(*[int(r) for r, _ in pts])
    ms = (C.c_double * len(pts))(*[float(t) for _, t in pts])
    out = (C.c_double * n)()
    check(lib.orch_speeds_from_profiles(n, npts, rows, ms, int(ref_rows), out))
    return list(out)


class DiTStep:
    """A library context for one DiT config: weights + workspace on the GPU."""

    def __init__(self, cfg, blob=None):
        self.cfg = cfg
        self._c = config_from(cfg)
        h = C.c_void_p()
        check(lib.orch_create(C.byref(self._c), C.byref(h)))
        self.handle = h
        if blob is not None:
            self.load(blob)

    def close(self):
        if getattr(self, "handle", None):
            lib.orch_destroy(self.handle)
            self.handle = None

    def __del__(self):
        self.close()

    def load(self, blob):
        import numpy as np
        b = np.ascontiguousarray(blob, dtype=np.uint8)
        check(lib.orch_load_dit_weights(self.handle, b.ctypes.data_as(C.c_void_p), b.nbytes))

    def stale_kv_bytes(self) -> int:
        return lib.orch_stale_kv_bytes(self.handle)

    def step(self, x_full, row_begin, row_end, t, t_prev, labels, cfg_scale, stale_kv,
             refresh, out_x, out_eps=None, z=None, eta=0.0, stream=None):
        lab = (C.c_int * len(labels))(*[int(v) for v in labels])
        check(lib.orch_patch_denoise_step(self.handle, _ptr(x_full), row_begin, row_end, t, t_prev,
                                          lab, float(cfg_scale), _ptr(stale_kv), int(refresh),
                                          _ptr(z), float(eta), _ptr(out_eps), _ptr(out_x),
                                          _stream(stream)))

    def sample_patch_parallel(self, latent, row_splits, tiers, t_grid, warmup, labels, cfg_scale,
                              kv_a, kv_b, stream=None):
        """Algorithm 1 on virtual devices (bands), in place on `latent`."""
        n = len(tiers)
        sp = (C.c_int * (n + 1))(*[int(v) for v in row_splits])
        tr = (C.c_int * n)(*[int(v) for v in tiers])
        tg = (C.c_int * len(t_grid))(*[int(v) for v in t_grid])
        lab = (C.c_int * len(labels))(*[int(v) for v in labels])
        check(lib.orch_sample_patch_parallel(self.handle, _ptr(latent), n, sp, tr, tg,
                                             len(t_grid) - 1, int(warmup), lab, float(cfg_scale),
                                             _ptr(kv_a), _ptr(kv_b), _stream(stream)))

    def set_work_split(self, enable: bool):
        check(lib.orch_set_work_split(self.handle, int(enable)))

    def set_kernel_timing(self, enable: bool):
        check(lib.orch_set_kernel_timing(self.handle, int(enable)))

    def kernel_times(self):
        """{class: (total_ms, launches)} since the last call (synchronises)."""
        ms = (C.c_double * len(KCLASSES))()
        n = (C.c_longlong * len(KCLASSES))()
        check(lib.orch_kernel_times(self.handle, ms, n))
        return {k: (ms[i], n[i]) for i, k in enumerate(KCLASSES)}

    def conditioning(self, t, labels, out, stream=None):
        lab = (C.c_int * len(labels))(*[int(v) for v in labels])
        check(lib.orch_op_conditioning(self.handle, t, lab, _ptr(out), _stream(stream)))

    def patch_embed(self, x_full, row_begin, row_end, out, stream=None):
        check(lib.orch_op_patch_embed(self.handle, _ptr(x_full), row_begin, row_end, _ptr(out),
                                      _stream(stream)))

    def final_layer(self, h, row_begin, row_end, mod, out_eps, stream=None):
        check(lib.orch_op_final_layer(self.handle, _ptr(h), row_begin, row_end, _ptr(mod),
                                      _ptr(out_eps), _stream(stream)))


def scheduler_update(x, eps_cond, eps_uncond, cfg_scale, z, a, b, c, out, stream=None):
    check(lib.orch_scheduler_update(_ptr(x), _ptr(eps_cond), _ptr(eps_uncond), float(cfg_scale),
                                    _ptr(z), a, b, c, _ptr(out), out.numel(), _stream(stream)))


def layernorm_modulate(x, rows, hidden, rows_per_batch, shift, scale, mod_stride, out, dtype,
                       stream=None):
    check(lib.orch_op_layernorm_modulate(_ptr(x), rows, hidden, rows_per_batch, _ptr(shift),
                                         _ptr(scale), mod_stride, _ptr(out), dtype,
                                         _stream(stream)))


def linear(A, M, K, W, N, bias, epilogue, gate, gate_stride, rows_per_batch, out, dtype,
           stream=None, workspace=None):
    ws_bytes = 0 if workspace is None else workspace.nbytes
    check(lib.orch_op_linear(_ptr(A), M, K, _ptr(W), N, _ptr(bias), epilogue, _ptr(gate),
                             gate_stride, rows_per_batch, _ptr(out), _ptr(workspace), ws_bytes,
                             dtype, _stream(stream)))


def linear_workspace_bytes(M, N, K, dtype) -> int:
    return lib.orch_linear_workspace_bytes(M, N, K, dtype)


def qkv_projection(A, B, n_tok, K, W, bias, hidden, heads, q_out, kv_out, kv_branch_stride,
                   kv_tokens, tok_offset, dtype, stream=None):
    check(lib.orch_op_qkv_projection(_ptr(A), B, n_tok, K, _ptr(W), _ptr(bias), hidden, heads,
                                     _ptr(q_out), _ptr(kv_out), kv_branch_stride, kv_tokens,
                                     tok_offset, dtype, _stream(stream)))


def attention_workspace_bytes(B, heads, n_q, n_kv, head_dim, dtype) -> int:
    return lib.orch_attention_workspace_bytes(B, heads, n_q, n_kv, head_dim, dtype)


def attention(q, kv_stale, stale_bs, kv_fresh, fresh_bs, fresh_begin, n_fresh, B, heads, n_q,
              n_kv, head_dim, out, dtype, workspace=None, stream=None):
    ws_bytes = 0 if workspace is None else workspace.nbytes
    check(lib.orch_op_attention(_ptr(q), _ptr(kv_stale), stale_bs, _ptr(kv_fresh), fresh_bs,
                                fresh_begin, n_fresh, B, heads, n_q, n_kv, head_dim, _ptr(out),
                                _ptr(workspace), ws_bytes, dtype, _stream(stream)))


def rotary_axes(channels, extent, theta=1e4, origin=(0.0, 0.0, 0.0), step=(1.0, 1.0, 1.0),
                interleaved=True) -> RotaryAxes:
    """Rotary positions of a (frames, rows, columns) grid, see orch_rotary_axes."""
    _check_ints(*channels, *extent)
    return RotaryAxes((C.c_int * 3)(*channels), (C.c_int * 3)(*extent), (C.c_double * 3)(*origin),
                      (C.c_double * 3)(*step), float(theta), int(interleaved))


_ROTARY_TENSOR = struct.Struct("=QQi4x6Q")     # RotaryTensor's layout


def rotary(axes: RotaryAxes, token_begin, x, out, stream=None):
    """Rotate x into out: tensors (or pairs of tensors, e.g. Q and K) [B, heads, n_tok, d] of any
    strides, their channels next to each other.  out may be x."""
    _check_ints(token_begin, 0)
    xs, outs = (x, out) if isinstance(x, (tuple, list)) else ((x,), (out,))
    B, _, n_tok, d = xs[0].shape
    dtype = xs[0].dtype
    if len(xs) != len(outs):
        raise OrchError(ORCH_EINVAL, "as many outputs as inputs are needed")
    ts, devices = b"", ()
    for a, o in zip(xs, outs):
        shape, sa, so = a.shape, a.stride(), o.stride()
        if o.shape != shape or a.dtype != dtype or o.dtype != dtype:
            raise OrchError(ORCH_EINVAL, "inputs and outputs must agree in shape and type")
        if shape[0] != B or shape[2] != n_tok or shape[3] != d or sa[3] != 1 or so[3] != 1:
            raise OrchError(ORCH_EINVAL, "tensors must be [B, heads, n_tok, d] with channels next to each other")
        devices += (a.get_device(), o.get_device())
        ts += _ROTARY_TENSOR.pack(a.data_ptr(), o.data_ptr(), shape[1], sa[0], sa[1], sa[2], so[0], so[1], so[2])
    code = _code(xs[0])
    check(lib.orch_op_rotary(C.byref(axes), ts, len(xs), B, n_tok, token_begin, d, code,
                             _stream_on(stream, *devices)))


def quantized_kv(values, exponents) -> QuantizedKV:
    """The 8-bit K/V cache held by two tensors: e4m3 (or uint8) values [B, 2, heads, tokens, d]
    and uint8 exponents [B, 2, heads, tokens], contiguous within a branch.  It keeps the tensors."""
    import torch
    B, two, heads, tokens, d = values.shape
    if two != 2 or tuple(exponents.shape) != (B, 2, heads, tokens):
        raise OrchError(ORCH_EINVAL, "values [B, 2, heads, tokens, d] and exponents [B, 2, heads, tokens] are needed")
    if values.dtype not in (torch.uint8, torch.float8_e4m3fn) or exponents.dtype != torch.uint8:
        raise OrchError(ORCH_EINVAL, "values must be e4m3fn or uint8, exponents uint8")
    if not (values[0].is_contiguous() and exponents[0].is_contiguous()):
        raise OrchError(ORCH_EINVAL, "a branch's values and exponents must be contiguous")
    c = QuantizedKV(values.data_ptr(), exponents.data_ptr(), values.stride(0), exponents.stride(0), tokens)
    c.tensors, c.devices = (values, exponents), (values.get_device(), exponents.get_device())
    c.shape = (B, heads, d)
    return c


def _check_cache(cache, B, heads, head_dim):
    b, h, d = cache.shape
    if heads != h or head_dim != d or B > b:
        raise OrchError(ORCH_EINVAL, f"{B} branches of {heads} heads of {head_dim} channels, the cache holds {b} of {h} of {d}")


def _check_buffer(name, t, dtype, elements, branch_stride=0):
    """t is of the code's type and holds `elements` elements from its first on, one behind the other within a branch."""
    if _code(t) != dtype:
        raise OrchError(ORCH_EINVAL, f"{name} is {t.dtype}, the call's type code {dtype}")
    if t.is_contiguous():
        held = t.numel()
    elif t.dim() > 1 and t.stride(0) == branch_stride and t[0].is_contiguous():
        held = (t.shape[0] - 1) * branch_stride + t[0].numel()
    else:
        raise OrchError(ORCH_EINVAL, f"{name} must be contiguous (a K/V buffer: within a branch)")
    if held < elements:
        raise OrchError(ORCH_EINVAL, f"{name} holds {held} elements, the call needs {elements}")


def _check_kv(name, kv, dtype, branch_stride, tokens, B, heads, head_dim):
    if branch_stride < 0:
        raise OrchError(ORCH_EINVAL, f"{name}: branch stride {branch_stride}")
    _check_buffer(name, kv, dtype, (B - 1) * branch_stride + 2 * tokens * heads * head_dim, branch_stride)


def kv_quantize(kv, kv_branch_stride, kv_tokens, kv_offset, cache: QuantizedKV, tok_offset, B, heads,
                n_tok, head_dim, dtype, stream=None):
    _check_cache(cache, B, heads, head_dim)
    _check_kv("kv", kv, dtype, kv_branch_stride, kv_tokens, B, heads, head_dim)
    _check_ints(kv_offset, tok_offset, n_tok, kv_tokens)
    st = _stream_on(stream, kv.get_device(), *cache.devices)
    check(lib.orch_op_kv_quantize(kv.data_ptr(), kv_branch_stride, kv_tokens, kv_offset, C.byref(cache),
                                  tok_offset, B, heads, n_tok, head_dim, dtype, st))


def kv_dequantize(cache: QuantizedKV, tok_offset, kv, kv_branch_stride, kv_tokens, kv_offset, B, heads,
                  n_tok, head_dim, dtype, stream=None):
    _check_cache(cache, B, heads, head_dim)
    _check_kv("kv", kv, dtype, kv_branch_stride, kv_tokens, B, heads, head_dim)
    _check_ints(kv_offset, tok_offset, n_tok, kv_tokens)
    st = _stream_on(stream, kv.get_device(), *cache.devices)
    check(lib.orch_op_kv_dequantize(C.byref(cache), tok_offset, kv.data_ptr(), kv_branch_stride, kv_tokens,
                                    kv_offset, B, heads, n_tok, head_dim, dtype, st))


def attention_quantized_workspace_bytes(B, heads, n_q, n_kv, head_dim, dtype) -> int:
    return lib.orch_attention_quantized_workspace_bytes(B, heads, n_q, n_kv, head_dim, dtype)


def attention_quantized_plan(B, heads, n_q, n_kv, head_dim, dtype, workspace_bytes):
    """(prepared, query_groups, key_parts) of a call, see orch_attention_quantized_plan."""
    r = [C.c_int() for _ in range(3)]
    check(lib.orch_attention_quantized_plan(B, heads, n_q, n_kv, head_dim, dtype, workspace_bytes, *map(C.byref, r)))
    return bool(r[0].value), r[1].value, r[2].value


def attention_quantized(q, cache: QuantizedKV, kv_fresh, fresh_bs, fresh_begin, n_fresh, B, heads, n_q,
                        head_dim, out, dtype, workspace=None, stream=None):
    _check_cache(cache, B, heads, head_dim)
    for name, t in (("q", q), ("out", out)):
        if t is not None:
            _check_buffer(name, t, dtype, B * n_q * heads * head_dim)
    if n_fresh > 0 and kv_fresh is not None:
        _check_kv("kv_fresh", kv_fresh, dtype, fresh_bs, n_fresh, B, heads, head_dim)
    _check_ints(n_q, fresh_begin, n_fresh)
    if workspace is not None and not workspace.is_contiguous():
        raise OrchError(ORCH_EINVAL, "workspace must be contiguous")
    ws_bytes = 0 if workspace is None else workspace.nbytes
    st = _stream_on(stream, *cache.devices, *[t.get_device() for t in (q, kv_fresh, out, workspace) if t is not None])
    check(lib.orch_op_attention_quantized(_ptr(q), C.byref(cache), _ptr(kv_fresh), fresh_bs, fresh_begin,
                                          n_fresh, B, heads, n_q, head_dim, _ptr(out), _ptr(workspace),
                                          ws_bytes, dtype, st))


def int8_rows(values, scales) -> Int8Rows:
    """int8 rows with a scale each, held by two tensors: int8 values [rows, cols], their columns next to
    each other and rows a multiple of 16 bytes apart, and fp32 scales [rows].  It keeps the tensors."""
    import torch
    rows, cols = values.shape
    if values.dtype != torch.int8 or scales.dtype != torch.float32:
        raise OrchError(ORCH_EINVAL, "values must be int8, scales fp32")
    if tuple(scales.shape) != (rows,) or not scales.is_contiguous():
        raise OrchError(ORCH_EINVAL, f"scales [{rows}] are needed, next to each other")
    if cols > 1 and values.stride(1) != 1:
        raise OrchError(ORCH_EINVAL, "a row's values must be next to each other")
    _check_ints(rows, cols)     # (the sizes of every call that takes them)
    r = Int8Rows(values.data_ptr(), scales.data_ptr(), values.stride(0))
    r.tensors, r.devices, r.shape = (values, scales), (values.get_device(), scales.get_device()), (rows, cols)
    r.ref, r.address = C.byref(r), C.addressof(r)
    return r


def norm(kind, eps=1e-6, weight=None, bias=None) -> Norm:
    """A norm ("none", "layer" or "rms") of block_norms, see orch_norm.  It keeps its fp32 [hidden] tensors."""
    import torch
    for t in (weight, bias):
        if t is not None and (t.dtype != torch.float32 or t.dim() != 1 or not t.is_contiguous()):
            raise OrchError(ORCH_EINVAL, "weight and bias must be fp32 [hidden], next to each other")
    if kind not in NORM_CODE:
        raise OrchError(ORCH_EINVAL, f"norm {kind!r}: one of {', '.join(NORM_CODE)} is needed")
    n = Norm(NORM_CODE[kind], eps, _ptr(weight), _ptr(bias))
    n.tensors = tuple(t for t in (weight, bias) if t is not None)
    n.devices, n.channels = tuple(t.get_device() for t in n.tensors), n.tensors[0].shape[0] if n.tensors else None
    if len(n.tensors) == 2 and bias.shape != weight.shape:
        raise OrchError(ORCH_EINVAL, "weight and bias must hold as many channels")
    n.packed = bytes(n)
    return n


_NO_NORM = Norm(0, 0.0, None, None)
_NO_NORM.devices, _NO_NORM.channels, _NO_NORM.packed = (), None, bytes(_NO_NORM)
_BLOCK_NORMS = struct.Struct("=24s24sf3i13Q")   # orch_block_norms' layout


_HERE = None            # torch's runtime functions, at the first use


def _stream_here(stream, device, *others):
    """_stream_on for tensors of one device: a current GPU that is theirs needs no second look."""
    global _HERE
    if device < 0 or stream is not None or others.count(device) != len(others):
        return _stream_on(stream, device, *others)
    if _HERE is None:
        from torch import _C
        _HERE = _C._cuda_getDevice, _C._cuda_getCurrentRawStream
    if _HERE[0]() != device:
        return _stream_on(stream, device)
    return _HERE[1](device)


def block_norms(h, y=None, h_out=None, out=None, *, post=None, pre=None, gate=None, shift=None, scale=None,
                rows_per_batch=0, residual_scale=1.0, stream=None):
    """The pass between two blocks, see orch_block_norms: h, h_out fp32 and y, out T [rows, hidden] with
    channels next to each other (out an Int8Rows: as codes), gate, shift and scale fp32 [branches, hidden]
    with one row stride, norms from norm().  What no block that ends (y) or follows (out) uses is ignored."""
    shape = h.shape
    rows, hidden = shape
    if y is None:
        post = gate = None
    if out is None:
        pre = shift = scale = None
        if h_out is None and rows:
            raise OrchError(ORCH_EINVAL, "nothing to write: h_out and out are None")
    post, pre = post or _NO_NORM, pre or _NO_NORM
    others = post.devices + pre.devices
    f32, one = _f32(), hidden == 1
    typed = y
    out8 = ptr_y = ptr_ho = ptr_o = st_y = st_ho = st_o = 0
    if out is not None:
        if type(out) is Int8Rows:
            if out.shape != (rows, hidden):
                raise OrchError(ORCH_EINVAL, f"out holds {out.shape} codes, the call writes {(rows, hidden)}")
            others += out.devices
            out8 = out.address
        else:
            st_o, c = out.stride()
            ptr_o = out.data_ptr()
            others += (out.get_device(),)
            if y is None:
                typed = out
            if out.shape != shape or out.dtype is not typed.dtype or not (c == 1 or one):
                _bad_rows(shape)
    st_h, c = h.stride()
    if h.dtype is not f32 or not (c == 1 or one):
        _bad_rows(shape)
    if y is not None:
        st_y, c = y.stride()
        ptr_y = y.data_ptr()
        others += (y.get_device(),)
        if y.shape != shape or not (c == 1 or one):
            _bad_rows(shape)
    if h_out is not None:
        st_ho, c = h_out.stride()
        ptr_ho = h_out.data_ptr()
        others += (h_out.get_device(),)
        if h_out.dtype is not f32 or h_out.shape != shape or not (c == 1 or one):
            _bad_rows(shape)
    code = ORCH_BF16 if typed is None else _code(typed)
    mods, mod_stride = [], None
    for t in (gate, shift, scale):
        if t is None:
            mods.append(0)
            continue
        (s, c), (branches, channels) = t.stride(), t.shape
        if mod_stride is None:
            mod_stride, need = s, -(-rows // rows_per_batch) if rows_per_batch > 0 else 0
        if branches < need or channels != hidden or t.dtype is not f32 or not (c == 1 or one) or (s != mod_stride and need > 1):
            raise OrchError(ORCH_EINVAL, f"gate, shift and scale must be fp32 [{need}, {hidden}] of one row stride, channels next to each other")
        others += (t.get_device(),)
        mods.append(t.data_ptr())
    if post.channels not in (None, hidden) or pre.channels not in (None, hidden):
        raise OrchError(ORCH_EINVAL, f"a norm's weight and bias must hold {hidden} channels")
    try:
        p = _BLOCK_NORMS.pack(post.packed, pre.packed, residual_scale, rows, hidden, rows_per_batch, h.data_ptr(), ptr_y, *mods,
                              ptr_ho, ptr_o, out8, st_h, st_y, mod_stride or 0, st_ho, st_o)
    except struct.error:
        _check_ints(rows, hidden, rows_per_batch)
        raise
    except OverflowError:
        raise OrchError(ORCH_EINVAL, f"residual_scale {residual_scale}: past fp32's range") from None
    rc = lib.orch_op_block_norms(p, code, _stream_here(stream, h.get_device(), *others))
    if rc:
        check(rc)


def _bad_rows(shape):
    raise OrchError(ORCH_EINVAL, f"h, y, h_out and out must be {list(shape)}, h and h_out fp32, y and out of one type, channels next to each other")


def quantize_rows(x, out: Int8Rows, stream=None):
    """Rows of x [rows, cols] (channels next to each other) to int8 with a scale each, see orch_op_quantize_rows."""
    rows, cols = x.shape
    st, c = x.stride()
    if out.shape != (rows, cols) or not (c == 1 or cols == 1):
        raise OrchError(ORCH_EINVAL, f"x must be {list(out.shape)}, as out, with channels next to each other")
    code = _code(x)
    rc = lib.orch_op_quantize_rows(x.data_ptr(), st, rows, cols, out.ref, code,
                                   _stream_here(stream, x.get_device(), *out.devices))
    if rc:
        check(rc)


def linear_quantized_workspace_bytes(M, N, K) -> int:
    _check_ints(M, N, K)
    return lib.orch_linear_quantized_workspace_bytes(M, N, K)


def _int8_operands(A, W, bias, workspace):
    """M, K, N, the workspace's bytes and the devices of a product."""
    (M, K), (N, k) = A.shape, W.shape
    if K != k:
        raise OrchError(ORCH_EINVAL, f"A has {K} channels, W {k}")
    devices = A.devices + W.devices
    if bias is not None:
        if bias.dtype is not _f32() or bias.shape != (N,) or not bias.is_contiguous():
            raise OrchError(ORCH_EINVAL, f"bias must be fp32 [{N}]")
        devices += (bias.get_device(),)
    ws_bytes = 0
    if workspace is not None:
        if not workspace.is_contiguous():
            raise OrchError(ORCH_EINVAL, "workspace must be contiguous")
        ws_bytes = workspace.nbytes
        devices += (workspace.get_device(),)
    return M, K, N, ws_bytes, devices


def linear_quantized(A: Int8Rows, W: Int8Rows, bias, epilogue, out, gate=None, rows_per_batch=0, workspace=None, stream=None):
    """A's rows times W's into out [M, N] (contiguous), see orch_op_linear_quantized; gate fp32 [branches, N]."""
    M, K, N, ws_bytes, devices = _int8_operands(A, W, bias, workspace)
    code = _code(out)
    if out.shape != (M, N) or not out.is_contiguous():
        raise OrchError(ORCH_EINVAL, f"out must be [{M}, {N}], contiguous")
    devices += (out.get_device(),)
    gate_stride = 0
    if not EPI_STORE <= epilogue <= EPI_RESIDUAL:
        _check_ints(epilogue, 0)
    if epilogue == EPI_RESIDUAL:
        _check_ints(rows_per_batch, 0)
        if code != ORCH_F32:
            raise OrchError(ORCH_EINVAL, "the residual epilogue adds to fp32")
        need = -(-M // max(1, rows_per_batch))
        if (gate is None or gate.dtype is not _f32() or gate.dim() != 2 or gate.shape[0] < need or gate.shape[1] != N
                or (N > 1 and gate.stride(1) != 1)):
            raise OrchError(ORCH_EINVAL, f"the residual epilogue needs gate, fp32 [{need}, {N}]")
        devices += (gate.get_device(),)
        gate_stride = gate.stride(0)
    rc = lib.orch_op_linear_quantized(A.ref, M, K, W.ref, N, _ptr(bias), epilogue, _ptr(gate), gate_stride, rows_per_batch,
                                      out.data_ptr(), _ptr(workspace), ws_bytes, code, _stream_here(stream, *devices))
    if rc:
        check(rc)


def qkv_projection_quantized(A: Int8Rows, W: Int8Rows, bias, q_out, kv_out, kv_tokens, tok_offset, workspace=None, stream=None):
    """Q [B, heads, n_tok, d] and the band's K and V of the K/V buffer kv_out [B, elements], see
    orch_op_qkv_projection_quantized."""
    M, K, N, ws_bytes, devices = _int8_operands(A, W, bias, workspace)
    B, heads, n_tok, d = q_out.shape
    code = _code(q_out)
    if B * n_tok != M or 3 * heads * d != N or not q_out.is_contiguous():
        raise OrchError(ORCH_EINVAL, f"q_out must be [B, heads, n_tok, d], contiguous, of {M} tokens and {N} / 3 channels")
    if kv_out.dim() != 2 or kv_out.shape[0] != B or kv_out.dtype is not q_out.dtype:
        raise OrchError(ORCH_EINVAL, f"kv_out must be [{B}, elements] of q_out's type")
    _check_ints(B, n_tok, kv_tokens, tok_offset)
    kv_bs, c = kv_out.stride()
    if kv_out.shape[1] < 2 * kv_tokens * heads * d or c != 1:
        raise OrchError(ORCH_EINVAL, f"kv_out must hold {2 * kv_tokens * heads * d} elements a branch, next to each other")
    devices += (q_out.get_device(), kv_out.get_device())
    rc = lib.orch_op_qkv_projection_quantized(A.ref, B, n_tok, K, W.ref, _ptr(bias), heads, d, q_out.data_ptr(),
                                              kv_out.data_ptr(), kv_bs, kv_tokens, tok_offset, _ptr(workspace), ws_bytes,
                                              code, _stream_here(stream, *devices))
    if rc:
        check(rc)


def unet_shape(cfg, eps: float = 1e-5) -> UNetConvShape:
    return UNetConvShape(cfg.height, cfg.width, cfg.channels, cfg.groups, cfg.out_channels, eps)


def unet_conv_workspace_bytes(shape: UNetConvShape, band_rows: int) -> int:
    return lib.orch_unet_conv_workspace_bytes(C.byref(shape), band_rows)


def unet_conv_band(shape: UNetConvShape, row_begin, row_end, x_band, gamma, beta, weight, bias,
                   stale_act, stale_sums, refresh, out, workspace, stream=None):
    ws_bytes = workspace.numel() * workspace.element_size()
    check(lib.orch_unet_conv_band(C.byref(shape), row_begin, row_end, _ptr(x_band), _ptr(gamma),
                                  _ptr(beta), _ptr(weight), _ptr(bias), _ptr(stale_act),
                                  _ptr(stale_sums), int(refresh), _ptr(out), _ptr(workspace),
                                  ws_bytes, _stream(stream)))
