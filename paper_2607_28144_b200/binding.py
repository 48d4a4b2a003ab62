"""Thin ctypes binding of the C ABI declared in ``include/regenvc_attn.h``.

Argument marshalling only: every step of the attention path runs in the CUDA
library.  PyTorch supplies device memory and streams.  If the shared library
is missing the first call raises; there is no CPU or library fallback.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libregenvc_attn.so")

OK, ERR_NULL_POINTER, ERR_BAD_SHAPE, ERR_UNSUPPORTED, ERR_MISALIGNED, ERR_ALIASING, ERR_CUDA, ERR_TIMEOUT, \
    ERR_WORKSPACE, ERR_RANGE, ERR_STATIC_LIMIT, ERR_INTERNAL = range(12)
STATIC_SCRATCH_BYTES = 16 << 20
NORM_NONE, NORM_LAYER, NORM_RMS = range(3)
TYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}

EXPORTS = [
    "regenvc_attn_forward", "regenvc_cross_attn_forward", "regenvc_attn_forward_host",
    "regenvc_cross_attn_forward_host", "regenvc_workspace_bytes", "regenvc_set_workspace",
    "regenvc_device_status", "regenvc_status_string", "regenvc_last_cuda_error", "regenvc_version",
    "regenvc_kernel_launch_count", "regenvc_shutdown", "regenvc_debug_set_phases",
    "regenvc_cross_attn_forward_static", "regenvc_static_device_status", "regenvc_attn_partial",
    "regenvc_prepared_bytes", "regenvc_cross_kv_prepare", "regenvc_cross_attn_forward_prepared",
    "regenvc_attn_forward_prepared", "regenvc_qkv_rope_project", "regenvc_out_project", "regenvc_attn_merge",
    "regenvc_ulysses_scatter_heads", "regenvc_ulysses_gather_heads", "regenvc_debug_expire_wait",
    "regenvc_block_norm_forward", "regenvc_block_norm_backward", "regenvc_block_norm_workspace_bytes",
    "regenvc_rope_axes", "regenvc_mxfp4_bytes", "regenvc_mxfp4_quantize", "regenvc_mxfp4_dequantize",
    "regenvc_mxfp4_project", "regenvc_mxfp4_linear", "regenvc_mxfp4_linear_scratch_bytes",
]


class BlockNormDesc(ctypes.Structure):
    """``regenvc_block_norm_desc``."""
    _fields_ = [(n, ctypes.c_int) for n in ("n_tokens", "channels", "tokens_per_mod", "x_type", "io_type", "norm",
                                            "post_norm")] + \
               [(n, ctypes.c_float) for n in ("eps", "post_eps", "residual_scale")] + \
               [(n, ctypes.c_longlong) for n in ("mod_stride", "x_stride", "y_stride", "x_out_stride", "h_stride",
                                                 "dx_out_stride", "dx_stride", "dy_stride")]


class RopeAxesDesc(ctypes.Structure):
    """``regenvc_rope_axes_desc``."""
    _fields_ = [(n, ctypes.c_int) for n in ("n_tokens", "n_q_heads", "n_k_heads", "head_dim", "type", "n_axes")] + \
               [("widths", ctypes.c_int * 4), ("rope_theta", ctypes.c_float)] + \
               [(n, ctypes.c_int) for n in ("halves", "whole_ladder", "pos_float", "inverse")] + \
               [(n, ctypes.c_longlong) for n in ("pos_stride", "q_token_stride", "q_head_stride", "k_token_stride",
                                                 "k_head_stride", "q_out_token_stride", "q_out_head_stride",
                                                 "k_out_token_stride", "k_out_head_stride")]


_lib = None


class RegenvcError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"regenvc status {code}: {text}")
        self.code = code


def lib() -> ctypes.CDLL:
    """Loads the CUDA shared library (built by ``python -m paper_2607_28144_b200.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2607_28144_b200.build` "
                           "(there is no fallback path)")
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, f32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
    L.regenvc_attn_forward.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, i32, f32, vp]
    L.regenvc_attn_forward.restype = i32
    L.regenvc_cross_attn_forward.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, vp]
    L.regenvc_cross_attn_forward.restype = i32
    L.regenvc_cross_attn_forward_static.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, vp]
    L.regenvc_cross_attn_forward_static.restype = i32
    L.regenvc_attn_partial.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, i32, i32, f32, vp]
    L.regenvc_attn_partial.restype = i32
    L.regenvc_attn_merge.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(vp), i32, vp, i32, i32, i32, vp]
    L.regenvc_attn_merge.restype = i32
    L.regenvc_ulysses_scatter_heads.argtypes = [vp, ctypes.POINTER(vp), i32, i32, i32, i32, i32, vp]
    L.regenvc_ulysses_scatter_heads.restype = i32
    L.regenvc_ulysses_gather_heads.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(i32), ctypes.POINTER(i32),
                                               i32, i32, i32, i32, i32, vp]
    L.regenvc_ulysses_gather_heads.restype = i32
    L.regenvc_attn_forward_host.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, i32, f32, vp]
    L.regenvc_attn_forward_host.restype = i32
    L.regenvc_cross_attn_forward_host.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, vp]
    L.regenvc_cross_attn_forward_host.restype = i32
    L.regenvc_prepared_bytes.argtypes = [i32, i32, i32]
    L.regenvc_prepared_bytes.restype = sz
    L.regenvc_cross_kv_prepare.argtypes = [vp, vp, vp, i32, i32, i32, vp]
    L.regenvc_cross_kv_prepare.restype = i32
    L.regenvc_cross_attn_forward_prepared.argtypes = [vp, vp, vp, i32, i32, i32, i32, vp]
    L.regenvc_cross_attn_forward_prepared.restype = i32
    L.regenvc_attn_forward_prepared.argtypes = [vp, vp, vp, i32, i32, i32, i32, vp]
    L.regenvc_attn_forward_prepared.restype = i32
    L.regenvc_qkv_rope_project.argtypes = [vp, vp, vp, vp, vp, f32, vp, vp, i32, i32, i32, i32, i32, f32, vp]
    L.regenvc_qkv_rope_project.restype = i32
    L.regenvc_out_project.argtypes = [vp, vp, vp, vp, i32, i32, i32, vp]
    L.regenvc_out_project.restype = i32
    i64 = ctypes.c_longlong
    L.regenvc_block_norm_forward.argtypes = [vp] * 12
    L.regenvc_block_norm_forward.restype = i32
    L.regenvc_block_norm_workspace_bytes.argtypes = [i32, i32]
    L.regenvc_block_norm_workspace_bytes.restype = sz
    L.regenvc_block_norm_backward.argtypes = [vp] * 19 + [sz, vp]
    L.regenvc_block_norm_backward.restype = i32
    L.regenvc_rope_axes.argtypes = [vp] * 7
    L.regenvc_rope_axes.restype = i32
    L.regenvc_mxfp4_bytes.argtypes = [i32, i32]
    L.regenvc_mxfp4_bytes.restype = sz
    L.regenvc_mxfp4_linear_scratch_bytes.argtypes = [i32, i32, i32]
    L.regenvc_mxfp4_linear_scratch_bytes.restype = sz
    L.regenvc_mxfp4_quantize.argtypes = [vp, i32, i32, i32, i64, vp, vp]
    L.regenvc_mxfp4_quantize.restype = i32
    L.regenvc_mxfp4_dequantize.argtypes = [vp, vp, i32, i32, i32, i64, vp]
    L.regenvc_mxfp4_dequantize.restype = i32
    L.regenvc_mxfp4_project.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, vp]
    L.regenvc_mxfp4_project.restype = i32
    L.regenvc_mxfp4_linear.argtypes = [vp, i32, i64, vp, vp, vp, i32, i32, i32, i32, vp, vp]
    L.regenvc_mxfp4_linear.restype = i32
    L.regenvc_workspace_bytes.argtypes = [i32, i32, i32]
    L.regenvc_workspace_bytes.restype = sz
    L.regenvc_set_workspace.argtypes = [vp, sz]
    L.regenvc_set_workspace.restype = i32
    L.regenvc_device_status.argtypes = [vp, ctypes.POINTER(i32)]
    L.regenvc_device_status.restype = i32
    L.regenvc_static_device_status.argtypes = [vp, ctypes.POINTER(i32)]
    L.regenvc_static_device_status.restype = i32
    L.regenvc_status_string.argtypes = [i32]
    L.regenvc_status_string.restype = ctypes.c_char_p
    L.regenvc_last_cuda_error.argtypes = []
    L.regenvc_last_cuda_error.restype = ctypes.c_char_p
    L.regenvc_version.argtypes = []
    L.regenvc_version.restype = ctypes.c_char_p
    L.regenvc_kernel_launch_count.argtypes = []
    L.regenvc_kernel_launch_count.restype = ctypes.c_ulonglong
    L.regenvc_debug_expire_wait.argtypes = [i32, vp]
    L.regenvc_debug_expire_wait.restype = i32
    L.regenvc_debug_set_phases.argtypes = [i32]
    L.regenvc_debug_set_phases.restype = i32
    L.regenvc_shutdown.argtypes = []
    L.regenvc_shutdown.restype = None
    _lib = L
    return L


def status_string(code: int) -> str:
    return lib().regenvc_status_string(code).decode()


def _check(code: int):
    if code != OK:
        text = status_string(code)
        if code == ERR_CUDA:
            text += ": " + lib().regenvc_last_cuda_error().decode()
        raise RegenvcError(code, text)


def _stream(stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream) if hasattr(stream, "cuda_stream") else int(stream)


def _dev_bf16(t: torch.Tensor, name: str):
    if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous() or t.dim() != 3:
        raise TypeError(f"{name} must be a contiguous CUDA bf16 tensor [tokens, heads, head_dim]")


def _host_bf16(t: torch.Tensor, name: str):
    if t.dtype != torch.bfloat16 or t.is_cuda or not t.is_contiguous() or t.dim() != 3:
        raise TypeError(f"{name} must be a contiguous CPU bf16 tensor [tokens, heads, head_dim]")


def regenvc_attn_forward(q, k, v, out, T: int, H: int, W: int, rope_theta: float = 10000.0, stream=None):
    """Self-attention with fused 3D RoPE on device tensors; asynchronous on ``stream``."""
    for t, nm in ((q, "q"), (k, "k"), (v, "v"), (out, "out")):
        _dev_bf16(t, nm)
    n, h, d = q.shape
    if n != T * H * W or k.shape != q.shape or v.shape != q.shape or out.shape != q.shape:
        raise ValueError("q, k, v, out must all be [T*H*W, heads, head_dim]")
    _check(lib().regenvc_attn_forward(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), T, H, W, h, d,
                                      float(rope_theta), _stream(stream)))
    return out


def regenvc_cross_attn_forward(q, k, v, out, stream=None):
    """Cross-attention of q [n_q, h, d] to k, v [n_kv, h, d] on device tensors."""
    for t, nm in ((q, "q"), (k, "k"), (v, "v"), (out, "out")):
        _dev_bf16(t, nm)
    n_q, h, d = q.shape
    n_kv = k.shape[0]
    if k.shape != (n_kv, h, d) or v.shape != k.shape or out.shape != q.shape:
        raise ValueError("shape mismatch")
    _check(lib().regenvc_cross_attn_forward(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), n_q, n_kv, h, d,
                                            _stream(stream)))
    return out


def regenvc_prepared_bytes(n_kv: int, n_heads: int, head_dim: int = 128) -> int:
    return int(lib().regenvc_prepared_bytes(n_kv, n_heads, head_dim))


def regenvc_cross_kv_prepare(k, v, prepared=None, stream=None):
    """Rewrites conditioning keys/values [n_kv, h, d] into operand form once; returns the ``prepared`` buffer
    (a CUDA uint8 tensor, allocated here with torch when not given) for regenvc_cross_attn_forward_prepared."""
    for t, nm in ((k, "k"), (v, "v")):
        _dev_bf16(t, nm)
    n_kv, h, d = k.shape
    if v.shape != k.shape:
        raise ValueError("shape mismatch")
    need = regenvc_prepared_bytes(n_kv, h, d)
    if prepared is None:
        prepared = torch.empty((need,), dtype=torch.uint8, device=k.device)
    if prepared.dtype != torch.uint8 or not prepared.is_cuda or prepared.numel() < need:
        raise TypeError(f"prepared must be a CUDA uint8 tensor of at least {need} bytes")
    _check(lib().regenvc_cross_kv_prepare(k.data_ptr(), v.data_ptr(), prepared.data_ptr(), n_kv, h, d, _stream(stream)))
    return prepared


def regenvc_cross_attn_forward_prepared(q, prepared, n_kv: int, out, stream=None):
    """Cross-attention of q [n_q, h, d] to the n_kv conditioning tokens whose operands are in ``prepared``."""
    _dev_bf16(q, "q")
    _dev_bf16(out, "out")
    n_q, h, d = q.shape
    if out.shape != q.shape:
        raise ValueError("shape mismatch")
    if prepared.dtype != torch.uint8 or not prepared.is_cuda or prepared.numel() < regenvc_prepared_bytes(n_kv, h, d):
        raise TypeError("prepared is too small for this shape")
    _check(lib().regenvc_cross_attn_forward_prepared(q.data_ptr(), prepared.data_ptr(), out.data_ptr(), n_q, n_kv, h, d,
                                                     _stream(stream)))
    return out


def regenvc_attn_forward_prepared(q_rot, prepared, n_kv: int, out, stream=None):
    """Attention on operands already in operand form: q_rot fp16 [n_q, h, d] (rotated), ``prepared`` = K' and V't."""
    if q_rot.dtype != torch.float16 or not q_rot.is_cuda or not q_rot.is_contiguous() or q_rot.dim() != 3:
        raise TypeError("q_rot must be a contiguous CUDA fp16 tensor [tokens, heads, head_dim]")
    _dev_bf16(out, "out")
    n_q, h, d = q_rot.shape
    if out.shape != q_rot.shape:
        raise ValueError("shape mismatch")
    if prepared.dtype != torch.uint8 or not prepared.is_cuda or prepared.numel() < regenvc_prepared_bytes(n_kv, h, d):
        raise TypeError("prepared is too small for this shape")
    _check(lib().regenvc_attn_forward_prepared(q_rot.data_ptr(), prepared.data_ptr(), out.data_ptr(), n_q, n_kv, h, d,
                                               _stream(stream)))
    return out


def regenvc_qkv_rope_project(x, w_qkv, b_qkv, g_q, g_k, eps: float, T: int, H: int, W: int, n_heads: int,
                             rope_theta: float = 10000.0, q_rot=None, prepared=None, stream=None):
    """QKV projection with fused RMS norm, rotation and operand layout.  x: CUDA bf16 [T*H*W, C]; w_qkv: CUDA bf16
    [3C, C]; b_qkv (fp32 [3C]), g_q, g_k (fp32 [C]) may be None.  Returns (q_rot fp16 [N, h, 128], prepared uint8),
    allocated here with torch when not given; feed them to regenvc_attn_forward_prepared."""
    if x.dtype != torch.bfloat16 or not x.is_cuda or not x.is_contiguous() or x.dim() != 2:
        raise TypeError("x must be a contiguous CUDA bf16 tensor [tokens, C]")
    n, C = x.shape
    if n != T * H * W or C != n_heads * 128:
        raise ValueError("x must be [T*H*W, n_heads * 128]")
    if w_qkv.dtype != torch.bfloat16 or not w_qkv.is_cuda or not w_qkv.is_contiguous() or tuple(w_qkv.shape) != (3 * C, C):
        raise TypeError("w_qkv must be a contiguous CUDA bf16 tensor [3C, C]")
    for t, nm, size in ((b_qkv, "b_qkv", 3 * C), (g_q, "g_q", C), (g_k, "g_k", C)):
        if t is not None and (t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous() or t.numel() != size):
            raise TypeError(f"{nm} must be a contiguous CUDA fp32 tensor of {size} elements (or None)")
    if q_rot is None:
        q_rot = torch.empty((n, n_heads, 128), dtype=torch.float16, device=x.device)
    need = regenvc_prepared_bytes(n, n_heads, 128)
    if prepared is None:
        prepared = torch.empty((need,), dtype=torch.uint8, device=x.device)
    if q_rot.dtype != torch.float16 or tuple(q_rot.shape) != (n, n_heads, 128) or not q_rot.is_contiguous():
        raise TypeError("q_rot must be a contiguous CUDA fp16 tensor [tokens, heads, 128]")
    if prepared.dtype != torch.uint8 or prepared.numel() < need:
        raise TypeError(f"prepared must be a CUDA uint8 tensor of at least {need} bytes")
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    _check(lib().regenvc_qkv_rope_project(x.data_ptr(), w_qkv.data_ptr(), ptr(b_qkv), ptr(g_q), ptr(g_k), float(eps),
                                          q_rot.data_ptr(), prepared.data_ptr(), T, H, W, n_heads, 128,
                                          float(rope_theta), _stream(stream)))
    return q_rot, prepared


def regenvc_out_project(attn_out, w_o, b_o, y=None, stream=None):
    """Output projection of the block: attn_out CUDA bf16 [tokens, heads, 128] (as the attention calls write it),
    w_o CUDA bf16 [C, C], b_o CUDA fp32 [C] or None.  Returns y bf16 [tokens, C] (allocated with torch if not given)."""
    _dev_bf16(attn_out, "attn_out")
    n, h, d = attn_out.shape
    C = h * d
    if w_o.dtype != torch.bfloat16 or not w_o.is_cuda or not w_o.is_contiguous() or tuple(w_o.shape) != (C, C):
        raise TypeError("w_o must be a contiguous CUDA bf16 tensor [C, C]")
    if b_o is not None and (b_o.dtype != torch.float32 or not b_o.is_cuda or not b_o.is_contiguous() or b_o.numel() != C):
        raise TypeError(f"b_o must be a contiguous CUDA fp32 tensor of {C} elements (or None)")
    if y is None:
        y = torch.empty((n, C), dtype=torch.bfloat16, device=attn_out.device)
    if y.dtype != torch.bfloat16 or not y.is_cuda or not y.is_contiguous() or tuple(y.shape) != (n, C):
        raise TypeError("y must be a contiguous CUDA bf16 tensor [tokens, C]")
    _check(lib().regenvc_out_project(attn_out.data_ptr(), w_o.data_ptr(), None if b_o is None else b_o.data_ptr(),
                                     y.data_ptr(), n, h, d, _stream(stream)))
    return y


# ---------------------------------------------------------------------------- steps around the attention of a block
_NORM_DESC, _ROPE_DESC = struct.Struct("@7i3f8q"), struct.Struct("@10if4i9q")   # the fields of the two descriptions
assert _NORM_DESC.size == ctypes.sizeof(BlockNormDesc) and _ROPE_DESC.size == ctypes.sizeof(RopeAxesDesc)


def _addr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _new(shape, dtype, device, stream):
    """A result or scratch tensor that belongs to the stream the call runs on."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(int(stream), device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _like(t, stream):
    """A packed result of an operand's shape and type."""
    if stream is None:
        return torch.empty_like(t) if t.is_contiguous() else torch.empty_like(t, memory_format=torch.contiguous_format)
    return _new(t.shape, t.dtype, t.device, stream)


def _place(first, *others) -> int:
    """All operands on the device the library launches on (the current one); returns its index."""
    if not first.is_cuda:
        raise TypeError("expected CUDA tensors")
    index = first.get_device()
    if index != torch.cuda.current_device():
        raise ValueError(f"operands are on cuda:{index}, the current device is cuda:{torch.cuda.current_device()}")
    for t in others:
        if t is not None and t.get_device() != index:
            raise ValueError("operands are on different devices")
    return index


def _launch_stream(stream, index: int) -> int:
    return torch._C._cuda_getCurrentRawStream(index) if stream is None else _stream(stream)


def _rows(t, name: str, dtype, n: int, c: int) -> int:
    """Checks a matrix and returns the elements between its rows as the library takes them (0: packed)."""
    if t.dtype is not dtype or t.shape != (n, c):
        raise TypeError(f"{name} must be {dtype} [{n}, {c}]")
    between, step = t.stride()
    if n > 1 and between >= c and (step == 1 or c == 1):   # the ordinary case, without a second call
        return between
    return _row_stride(t, name)


def _row_stride(t, name: str = "the tensor") -> int:
    """Elements between rows as the library takes them (0: packed); rows that share memory are refused here, since an
    expanded tensor's stride of 0 would read as "packed"."""
    if t is None:
        return 0
    rows, cols = t.shape
    between, step = t.stride()
    if step != 1 and cols > 1:
        raise TypeError(f"{name} must have neighbouring columns")
    if rows < 2:
        return 0
    if between < cols:
        raise ValueError(f"{name} has rows that overlap (an expanded tensor?)")
    return between


def _vector(t, name: str, size: int):
    if t is not None and (t.dtype is not torch.float32 or t.numel() != size or not t.is_contiguous()):
        raise TypeError(f"{name} must be a contiguous fp32 tensor of {size} elements (or None)")


def _modulation(n: int, c: int, tokens_per_mod, gate, scale, shift):
    """Checks the modulation tables and returns (tokens_per_mod, rows, row stride)."""
    most = max(n, 1)   # (no tokens at all: the library refuses that)
    per = most if tokens_per_mod is None else min(int(tokens_per_mod), most)
    if per < 1:
        raise ValueError("tokens_per_mod must be at least 1")
    rows = -(-n // per)
    stride = 0
    for t, name in ((gate, "gate"), (scale, "scale"), (shift, "shift")):
        if t is not None:
            s = _rows(t, name, torch.float32, rows, c)
            if stride and s != stride:
                raise ValueError("gate, scale and shift must have the same distance between rows")
            stride = s
    return per, rows, stride


def regenvc_block_norm_forward(x, y=None, *, gate=None, post_norm: int = NORM_NONE, post_weight=None,
                               post_eps: float = 1e-6, residual_scale: float = 1.0, norm: int = NORM_LAYER, weight=None,
                               bias=None, eps: float = 1e-6, scale=None, shift=None, tokens_per_mod=None, h_dtype=None,
                               x_out=None, h=None, stream=None):
    """x' = residual_scale x + gate N2(y) post_weight and h = (N1(x') weight + bias) (1 + scale) + shift in one pass (N2(y)
    is y where post_norm is NORM_NONE); returns (x' or None where y is None, h or None where norm is NORM_NONE).  x [tokens, C]: bf16, fp16 or fp32; y and h: the
    same type, or any of them where x is fp32 (h: ``h_dtype``, else y's, else x's).  gate, scale, shift: fp32 [rows, C],
    one row per ``tokens_per_mod`` tokens (None: one for all); post_weight, weight, bias: fp32 [C].  x may be given as
    ``x_out`` (in place)."""
    if x.dim() != 2 or x.dtype not in TYPES:
        raise TypeError("x must be [tokens, C] in bf16, fp16 or fp32")
    index = _place(x, y, gate, post_weight, weight, bias, scale, shift, x_out, h)
    n, c = x.shape
    io = h.dtype if h is not None else h_dtype or (y.dtype if y is not None else x.dtype)
    if io not in TYPES:
        raise TypeError("h must be bf16, fp16 or fp32")
    x_stride = _row_stride(x, "x")
    y_stride = 0 if y is None else _rows(y, "y", io, n, c)
    if post_weight is not None:
        _vector(post_weight, "post_weight", c)
    if weight is not None:
        _vector(weight, "weight", c)
    if bias is not None:
        _vector(bias, "bias", c)
    per, _, mod_stride = _modulation(n, c, tokens_per_mod, gate, scale, shift)
    x_out_stride = h_stride = 0
    if x_out is not None:
        if y is None:
            raise ValueError("x_out needs y")
        x_out_stride = _rows(x_out, "x_out", x.dtype, n, c)
    elif y is not None:
        x_out = _like(x, stream)
    if h is not None:
        if norm == NORM_NONE:
            raise ValueError("h needs a norm")
        h_stride = _rows(h, "h", io, n, c)
    elif norm != NORM_NONE:
        h = _like(x, stream) if io is x.dtype else _new((n, c), io, x.device, stream)
    d = _NORM_DESC.pack(n, c, per, TYPES[x.dtype], TYPES[io], norm, post_norm, eps, post_eps, residual_scale,
                        mod_stride, x_stride, y_stride, x_out_stride, h_stride, 0, 0, 0)
    _check(lib().regenvc_block_norm_forward(d, x.data_ptr(), _addr(y), _addr(gate), _addr(post_weight), _addr(weight),
                                            _addr(bias), _addr(scale), _addr(shift), _addr(x_out), _addr(h),
                                            _launch_stream(stream, index)))
    return x_out, h


def regenvc_block_norm_workspace_bytes(n_tokens: int, channels: int) -> int:
    return int(lib().regenvc_block_norm_workspace_bytes(n_tokens, channels))


def regenvc_block_norm_backward(dh, x_out, *, dx_out=None, y=None, gate=None, post_norm: int = NORM_NONE, post_weight=None,
                                post_eps: float = 1e-6, residual_scale: float = 1.0, norm: int = NORM_LAYER, weight=None,
                                bias=None, eps: float = 1e-6, scale=None, shift=None, tokens_per_mod=None, dx=None,
                                workspace=None, stream=None):
    """Gradients of regenvc_block_norm_forward at the saved ``x_out`` (its x where y was None): dh is the gradient of h
    (None where norm is NORM_NONE), dx_out the one that reaches x_out by other ways (or None).  Returns a dict: dx, dy
    (None without y), and dgate, dpost_weight, dweight, dbias, dscale, dshift, each None where its parameter is.  ``shift``
    only says whether dshift is wanted.  ``dx`` may be dx_out (in place)."""
    like = x_out if x_out is not None else dx_out
    if like is None or like.dim() != 2 or like.dtype not in TYPES:
        raise TypeError("x_out must be [tokens, C] in bf16, fp16 or fp32")
    index = _place(like, x_out, dh, dx_out, y, gate, post_weight, weight, bias, scale, shift, dx, workspace)
    n, c = like.shape
    io = dh.dtype if dh is not None else (y.dtype if y is not None else like.dtype)
    if io not in TYPES:
        raise TypeError("dh must be bf16, fp16 or fp32")
    y_stride = 0 if y is None else _rows(y, "y", io, n, c)
    x_stride = 0 if x_out is None else _rows(x_out, "x_out", like.dtype, n, c)
    h_stride = 0 if dh is None else _rows(dh, "dh", io, n, c)
    more_stride = 0 if dx_out is None else _rows(dx_out, "dx_out", like.dtype, n, c)
    if post_weight is not None:
        _vector(post_weight, "post_weight", c)
    if weight is not None:
        _vector(weight, "weight", c)
    if bias is not None:
        _vector(bias, "bias", c)
    per, _, mod_stride = _modulation(n, c, tokens_per_mod, gate, scale, shift)
    if dx is None:
        dx, dx_stride = _like(like, stream), 0
    else:
        dx_stride = _rows(dx, "dx", like.dtype, n, c)
    # every parameter's gradient has its shape, packed
    dy = None if y is None else _like(y, stream)
    dgate = None if gate is None else _like(gate, stream)
    dscale = None if scale is None else _like(scale, stream)
    dshift = None if shift is None else _like(shift, stream)
    dpost = None if post_weight is None else _like(post_weight, stream)
    dweight = None if weight is None else _like(weight, stream)
    dbias = None if bias is None else _like(bias, stream)
    if workspace is None:
        workspace = _new((regenvc_block_norm_workspace_bytes(n, c),), torch.uint8, like.device, stream)
    d = _NORM_DESC.pack(n, c, per, TYPES[like.dtype], TYPES[io], norm, post_norm, eps, post_eps, residual_scale,
                        mod_stride, 0, y_stride, x_stride, h_stride, more_stride, dx_stride, 0)
    _check(lib().regenvc_block_norm_backward(
        d, _addr(x_out), _addr(y), _addr(gate), _addr(post_weight), _addr(weight), _addr(bias), _addr(scale),
        _addr(dh), _addr(dx_out), dx.data_ptr(), _addr(dy), _addr(dgate), _addr(dpost), _addr(dweight), _addr(dbias),
        _addr(dscale), _addr(dshift), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
        _launch_stream(stream, index)))
    return {"dx": dx, "dy": dy, "dgate": dgate, "dscale": dscale, "dshift": dshift, "dpost_weight": dpost,
            "dweight": dweight, "dbias": dbias}


def regenvc_rope_axes(q, k, positions, widths, *, rope_theta: float = 10000.0, halves: bool = False,
                      whole_ladder: bool = False, inverse: bool = False, q_out=None, k_out=None, stream=None):
    """Rotates q [tokens, heads, head_dim] and k (fewer heads allowed, or None) by ``positions`` [axes, tokens] (int32 or
    fp32), ``widths[a]`` elements of a head turning with axis a; returns (q_out, k_out).  Views with any token and head
    strides are taken as they are; q / k given as q_out / k_out are rotated in place.  ``inverse`` turns back, which is the
    gradient."""
    if q.dim() != 3 or q.dtype not in TYPES:
        raise TypeError("q must be [tokens, heads, head_dim] in bf16, fp16 or fp32")
    index = _place(q, k, positions, q_out, k_out)
    n, hq, d = q.shape
    widths = list(widths)
    if positions.dtype not in (torch.int32, torch.float32) or positions.shape != (len(widths), n) or \
            (n > 1 and positions.stride(1) != 1) or (len(widths) > 1 and positions.stride(0) < n):
        raise TypeError(f"positions must be int32 or fp32 [{len(widths)}, {n}] with neighbouring tokens")
    if k is not None and (k.dtype != q.dtype or k.dim() != 3 or k.shape[0] != n or k.shape[2] != d):
        raise TypeError("k must be [tokens, heads, head_dim] of q's type")
    if k is None and k_out is not None:
        raise ValueError("k_out needs k")
    if not 1 <= len(widths) <= 4:
        raise RegenvcError(ERR_BAD_SHAPE, status_string(ERR_BAD_SHAPE))
    if q_out is None:
        q_out = _like(q, stream)
    if k is not None and k_out is None:
        k_out = _like(k, stream)
    hk = 0 if k is None else k.shape[1]
    strides = []
    for t, like, name in ((q, q, "q"), (k, k, "k"), (q_out, q, "q_out"), (k_out, k, "k_out")):
        if t is None:
            strides += [0, 0]
            continue
        if t.is_contiguous() and t.dtype is q.dtype and t.shape == like.shape:
            strides += [0, 0]
            continue
        token, head, step = t.stride()
        heads = t.shape[1]
        if t.dtype is not q.dtype or t.shape != like.shape or (d > 1 and step != 1):
            raise TypeError(f"{name} must have its operand's type and shape and neighbouring elements of a head")
        if (n > 1 and token < d) or (heads > 1 and head < d):
            raise ValueError(f"{name} has vectors that overlap (an expanded tensor?)")
        # the stride of an axis with one entry is never used: name the packed one
        head = head if heads > 1 else d
        strides += [token if n > 1 else heads * head, head]
    desc = _ROPE_DESC.pack(n, hq, hk, d, TYPES[q.dtype], len(widths), *(widths + [0, 0, 0])[:4], rope_theta, bool(halves),
                           bool(whole_ladder), positions.dtype is torch.float32, bool(inverse),
                           positions.stride(0) if len(widths) > 1 else 0, *strides)
    _check(lib().regenvc_rope_axes(desc, q.data_ptr(), _addr(k), positions.data_ptr(), q_out.data_ptr(),
                                   _addr(k_out), _launch_stream(stream, index)))
    return q_out, k_out


def regenvc_mxfp4_bytes(rows: int, cols: int) -> int:
    return int(lib().regenvc_mxfp4_bytes(rows, cols))


def _mx_bytes(rows: int, cols: int) -> int:
    """regenvc_mxfp4_bytes() without the call, for sizes the library then checks itself."""
    blocks = -(-cols // 128)
    return -(-rows * blocks // 8) * 512 + -(-rows // 128) * blocks * 512


def _mx_packed(t, name: str, rows: int, cols: int):
    need = _mx_bytes(rows, cols)
    if t.dtype is not torch.uint8 or t.numel() < need or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous uint8 tensor of at least {need} bytes")


def _mx_values(t, name: str) -> int:
    if t.dim() != 2 or t.dtype not in TYPES:
        raise TypeError(f"{name} must be [rows, cols] in bf16, fp16 or fp32")
    return _row_stride(t, name)


def regenvc_mxfp4_quantize(src, packed=None, stream=None):
    """Rows of bf16, fp16 or fp32 [rows, cols] to microscaled 4-bit form; returns the ``packed`` uint8 tensor."""
    stride = _mx_values(src, "src")
    index = _place(src, packed)
    rows, cols = src.shape
    if packed is None:
        packed = _new((_mx_bytes(rows, cols),), torch.uint8, src.device, stream)
    else:
        _mx_packed(packed, "packed", rows, cols)
    _check(lib().regenvc_mxfp4_quantize(src.data_ptr(), TYPES[src.dtype], rows, cols, stride, packed.data_ptr(),
                                        _launch_stream(stream, index)))
    return packed


def regenvc_mxfp4_dequantize(packed, rows: int, cols: int, dtype=torch.bfloat16, out=None, stream=None):
    """The [rows, cols] values that a packed matrix stands for."""
    _mx_packed(packed, "packed", rows, cols)
    index = _place(packed, out)
    if out is None:
        out = _new((rows, cols), dtype, packed.device, stream)
    stride = _mx_values(out, "out")
    if out.shape != (rows, cols):
        raise TypeError(f"out must be [{rows}, {cols}]")
    _check(lib().regenvc_mxfp4_dequantize(packed.data_ptr(), out.data_ptr(), TYPES[out.dtype], rows, cols, stride,
                                          _launch_stream(stream, index)))
    return out


def regenvc_mxfp4_linear_scratch_bytes(n_tokens: int, out_features: int, in_features: int) -> int:
    return int(lib().regenvc_mxfp4_linear_scratch_bytes(n_tokens, out_features, in_features))


def _mx_result(y, y_dtype, n: int, features: int, device, stream):
    if (y_dtype if y is None else y.dtype) not in (torch.bfloat16, torch.float16):
        raise TypeError("y must be bf16 or fp16")
    if y is None:
        return _new((n, features), y_dtype, device, stream)
    if y.shape != (n, features) or not y.is_contiguous():
        raise TypeError(f"y must be a contiguous tensor [{n}, {features}]")
    return y


def regenvc_mxfp4_project(x_packed, w_packed, n_tokens: int, out_features: int, in_features: int, bias=None, *,
                          y_dtype=torch.bfloat16, y=None, stream=None):
    """y [n_tokens, out_features] = x w^T + bias on packed 4-bit x [n_tokens, in_features] and w [out_features,
    in_features]; bias fp32 [out_features] or None."""
    _mx_packed(x_packed, "x_packed", n_tokens, in_features)
    _mx_packed(w_packed, "w_packed", out_features, in_features)
    _vector(bias, "bias", out_features)
    index = _place(x_packed, w_packed, bias, y)
    y = _mx_result(y, y_dtype, n_tokens, out_features, x_packed.device, stream)
    _check(lib().regenvc_mxfp4_project(x_packed.data_ptr(), w_packed.data_ptr(), _addr(bias), y.data_ptr(), TYPES[y.dtype],
                                       n_tokens, out_features, in_features, _launch_stream(stream, index)))
    return y


def regenvc_mxfp4_linear(x, w_packed, out_features: int, bias=None, *, y_dtype=torch.bfloat16, y=None, scratch=None,
                         stream=None):
    """y [tokens, out_features] = Q(x) w^T + bias: x [tokens, in_features] (bf16, fp16 or fp32) is taken to 4 bits in the
    call, w is packed (regenvc_mxfp4_quantize).  ``scratch``: uint8, regenvc_mxfp4_linear_scratch_bytes() long."""
    stride = _mx_values(x, "x")
    n, cols = x.shape
    _mx_packed(w_packed, "w_packed", out_features, cols)
    _vector(bias, "bias", out_features)
    index = _place(x, w_packed, bias, y, scratch)
    y = _mx_result(y, y_dtype, n, out_features, x.device, stream)
    need = regenvc_mxfp4_linear_scratch_bytes(n, out_features, cols)
    if scratch is None and need:
        scratch = _new((need,), torch.uint8, x.device, stream)
    if scratch is not None and (scratch.dtype != torch.uint8 or not scratch.is_contiguous() or scratch.numel() < need):
        raise TypeError(f"scratch must be a contiguous uint8 tensor of at least {need} bytes")
    _check(lib().regenvc_mxfp4_linear(x.data_ptr(), TYPES[x.dtype], stride, w_packed.data_ptr(), _addr(bias),
                                      y.data_ptr(), TYPES[y.dtype], n, out_features, cols, _addr(scratch),
                                      _launch_stream(stream, index)))
    return y


def regenvc_cross_attn_forward_static(q, k, v, out, stream=None):
    """Cross-attention without any device allocation by the library (for callers in a real-time loop, or
    in a process whose memory pool owns the GPU): the operand scratch is a fixed 16 MiB array inside the
    library, shared by all calls on the device, so calls must not overlap on the GPU; shapes with
    n_heads * ceil(n_kv / 128) * 128 > 32768 raise ERR_STATIC_LIMIT."""
    for t, nm in ((q, "q"), (k, "k"), (v, "v"), (out, "out")):
        _dev_bf16(t, nm)
    n_q, h, d = q.shape
    n_kv = k.shape[0]
    if k.shape != (n_kv, h, d) or v.shape != k.shape or out.shape != q.shape:
        raise ValueError("shape mismatch")
    _check(lib().regenvc_cross_attn_forward_static(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), n_q,
                                                   n_kv, h, d, _stream(stream)))
    return out


def regenvc_attn_partial(q, k, v, o_part, ml, T: int, H: int, W: int, q_token0: int, kv_token0: int,
                         rope_theta: float = 10000.0, stream=None):
    """Unnormalised attention of the query tokens q_token0.. against the key/value block kv_token0.. of the grid.
    o_part: CUDA fp32 [n_q, h, d]; ml: CUDA fp32 [n_q, h, 2] (reference, row sum)."""
    for t, nm in ((q, "q"), (k, "k"), (v, "v")):
        _dev_bf16(t, nm)
    n_q, h, d = q.shape
    n_kv = k.shape[0]
    if k.shape != (n_kv, h, d) or v.shape != k.shape:
        raise ValueError("shape mismatch")
    if o_part.dtype != torch.float32 or tuple(o_part.shape) != (n_q, h, d) or not o_part.is_contiguous():
        raise TypeError("o_part must be a contiguous CUDA fp32 tensor [n_q, heads, head_dim]")
    if ml.dtype != torch.float32 or tuple(ml.shape) != (n_q, h, 2) or not ml.is_contiguous():
        raise TypeError("ml must be a contiguous CUDA fp32 tensor [n_q, heads, 2]")
    _check(lib().regenvc_attn_partial(q.data_ptr(), k.data_ptr(), v.data_ptr(), o_part.data_ptr(), ml.data_ptr(),
                                      T, H, W, q_token0, n_q, kv_token0, n_kv, h, d, float(rope_theta),
                                      _stream(stream)))
    return o_part, ml


def regenvc_attn_merge(o_parts, mls, out, stream=None):
    """Merges partial results of several key/value blocks (same query range) into bf16 ``out`` [n_q, h, d]."""
    _dev_bf16(out, "out")
    n_q, h, d = out.shape
    n = len(o_parts)
    if n != len(mls):
        raise ValueError("need one (m, l) tensor per partial result")
    arr_o = (ctypes.c_void_p * n)(*[t.data_ptr() for t in o_parts])
    arr_m = (ctypes.c_void_p * n)(*[t.data_ptr() for t in mls])
    _check(lib().regenvc_attn_merge(arr_o, arr_m, n, out.data_ptr(), n_q, h, d, _stream(stream)))
    return out


def _ptr(x) -> int:
    return x.data_ptr() if isinstance(x, torch.Tensor) else int(x)


def regenvc_ulysses_scatter_heads(x_local, dst, dst_token0: int, stream=None):
    """Head-group r of this GPU's tokens ``x_local`` [n_local, h, d] goes to ``dst[r]`` [group tokens, h/len(dst), d]
    at rows ``dst_token0``...  ``dst`` holds CUDA tensors or raw device addresses (a peer GPU's mapped buffer)."""
    _dev_bf16(x_local, "x_local")
    n, h, d = x_local.shape
    world = len(dst)
    arr = (ctypes.c_void_p * world)(*[_ptr(t) for t in dst])
    _check(lib().regenvc_ulysses_scatter_heads(x_local.data_ptr(), arr, world, n, int(dst_token0), h, d,
                                               _stream(stream)))


def regenvc_ulysses_gather_heads(x_heads, dst, token0, n_tokens, n_heads_dst: int, dst_head0: int, stream=None):
    """Tokens ``token0[r]``.. (``n_tokens[r]`` of them) of this GPU's heads ``x_heads`` [tokens, h_local, d] go to
    ``dst[r]`` [n_tokens[r], n_heads_dst, d] at heads ``dst_head0``...  ``dst`` as in the scatter call."""
    _dev_bf16(x_heads, "x_heads")
    _, h_loc, d = x_heads.shape
    world = len(dst)
    if len(token0) != world or len(n_tokens) != world:
        raise ValueError("need one token range per destination")
    if any(t0 < 0 or n < 0 or t0 + n > x_heads.shape[0] for t0, n in zip(token0, n_tokens)):
        raise ValueError("token range outside x_heads")
    arr = (ctypes.c_void_p * world)(*[_ptr(t) for t in dst])
    a0 = (ctypes.c_int * world)(*[int(x) for x in token0])
    an = (ctypes.c_int * world)(*[int(x) for x in n_tokens])
    _check(lib().regenvc_ulysses_gather_heads(x_heads.data_ptr(), arr, a0, an, world, h_loc, int(n_heads_dst),
                                              int(dst_head0), d, _stream(stream)))


def regenvc_attn_forward_host(q, k, v, out, T: int, H: int, W: int, rope_theta: float = 10000.0, stream=None):
    """Same operation with all four tensors in host memory (copies inside the call; returns when done)."""
    for t, nm in ((q, "q"), (k, "k"), (v, "v"), (out, "out")):
        _host_bf16(t, nm)
    n, h, d = q.shape
    if n != T * H * W or k.shape != q.shape or v.shape != q.shape or out.shape != q.shape:
        raise ValueError("q, k, v, out must all be [T*H*W, heads, head_dim]")
    _check(lib().regenvc_attn_forward_host(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), T, H, W, h, d,
                                           float(rope_theta), _stream(stream)))
    return out


def regenvc_cross_attn_forward_host(q, k, v, out, stream=None):
    for t, nm in ((q, "q"), (k, "k"), (v, "v"), (out, "out")):
        _host_bf16(t, nm)
    n_q, h, d = q.shape
    n_kv = k.shape[0]
    if k.shape != (n_kv, h, d) or v.shape != k.shape or out.shape != q.shape:
        raise ValueError("shape mismatch")
    _check(lib().regenvc_cross_attn_forward_host(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), n_q, n_kv,
                                                 h, d, _stream(stream)))
    return out


def regenvc_workspace_bytes(n_kv: int, n_heads: int, head_dim: int = 128) -> int:
    return int(lib().regenvc_workspace_bytes(n_kv, n_heads, head_dim))


def regenvc_set_workspace(buf: Optional[torch.Tensor]):
    """Use ``buf`` (a CUDA uint8 tensor the caller keeps alive) as this thread's workspace; None resets."""
    if buf is None:
        _check(lib().regenvc_set_workspace(None, 0))
    else:
        _check(lib().regenvc_set_workspace(buf.data_ptr(), buf.numel() * buf.element_size()))


def regenvc_device_status(stream=None) -> int:
    """Waits for ``stream`` and returns (then clears) the sticky device status."""
    st = ctypes.c_int(0)
    _check(lib().regenvc_device_status(_stream(stream), ctypes.byref(st)))
    return st.value


def regenvc_static_device_status(stream=None) -> int:
    """Waits for ``stream`` and returns (then clears) the status word of the allocation-free entry point."""
    st = ctypes.c_int(0)
    _check(lib().regenvc_static_device_status(_stream(stream), ctypes.byref(st)))
    return st.value


def regenvc_version() -> str:
    return lib().regenvc_version().decode()


def regenvc_kernel_launch_count() -> int:
    return int(lib().regenvc_kernel_launch_count())


def regenvc_debug_set_phases(mask: int):
    """Profiling aid: 1 = preparation pass only, 2 = attention kernel only, 3 = both (default); + 4: no persistent
    form for short key sequences; + 8 / + 16: always / never the kernel on pairs of thread blocks; + 32: always that
    kernel, on a grid of two pairs that walk over all work items."""
    _check(lib().regenvc_debug_set_phases(mask))


def regenvc_debug_expire_wait(limit_us: int = 500, stream=None):
    """Test aid: one warp waits limit_us on a barrier nothing completes; the sticky status becomes ERR_TIMEOUT."""
    _check(lib().regenvc_debug_expire_wait(int(limit_us), _stream(stream)))


def regenvc_shutdown():
    lib().regenvc_shutdown()
