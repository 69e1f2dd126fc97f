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
