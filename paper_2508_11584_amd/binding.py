"""ctypes binding of the C ABI declared in include/vpe.h (same names, argument marshalling only).

There is no fallback: if libvpe.so is missing it is built with hipcc, and if that fails the
import of the library raises.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from struct import Struct, error as StructError
from typing import List, Optional, Sequence

import numpy as np

VPE_OK, VPE_SKIPPED, VPE_BUSY, VPE_EINVAL, VPE_ENOMEM, VPE_ESTALE, VPE_EHIP = 0, 1, 2, -1, -2, -3, -4
VPE_F32, VPE_BF16 = 0, 1
VPE_MLP_GELU, VPE_MLP_SWIGLU = 0, 1
VPE_HEAD_SEG, VPE_HEAD_DEPTH, VPE_HEAD_DET, VPE_HEAD_DPT, VPE_HEAD_QUERY = 0, 1, 2, 3, 4
VPE_NORM_NONE, VPE_NORM_LAYER, VPE_NORM_RMS = 0, 1, 2
VPE_FLAG_GRAPHS, VPE_FLAG_HOST_ONLY, VPE_FLAG_WALL_CLOCK, VPE_FLAG_TIMING = 1, 2, 4, 8

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libvpe.so")
_lib = None


class vpe_feat(C.Structure):
    _fields_ = [("slot", C.c_int32), ("reserved", C.c_int32), ("frame", C.c_int64)]


class vpe_backbone_cfg(C.Structure):
    _fields_ = [("dim", C.c_int32), ("depth", C.c_int32), ("heads", C.c_int32), ("mlp_hidden", C.c_int32),
                ("mlp_kind", C.c_int32), ("registers", C.c_int32), ("img_h", C.c_int32), ("img_w", C.c_int32),
                ("batch", C.c_int32), ("dtype", C.c_int32), ("taps", C.c_int32 * 4), ("ring_slots", C.c_int32),
                ("flags", C.c_int32), ("ln_eps", C.c_float), ("encoder_lanes", C.c_int32), ("head_streams", C.c_int32),
                ("reserved", C.c_int32), ("weights", C.c_void_p),
                ("weights_bytes", C.c_uint64)]


class vpe_head_cfg(C.Structure):
    _fields_ = [("kind", C.c_int32), ("classes", C.c_int32), ("channels", C.c_int32), ("every_n", C.c_int32),
                ("weights", C.c_void_p), ("weights_bytes", C.c_uint64)]


class vpe_attention_args(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "heads", "kv_heads", "head_dim", "sequences", "max_q", "max_k", "q_rows", "k_rows", "causal")] + \
               [("scale", C.c_float), ("cap", C.c_float)] + [(n, C.c_void_p) for n in ("q", "k", "v", "out")] + \
               [(n, C.c_int64) for n in ("q_row", "q_head", "k_row", "k_head", "v_row", "v_head", "out_row", "out_head")] + \
               [(n, C.c_void_p) for n in ("q_offsets", "k_offsets", "k_lengths", "prefix", "slopes", "q_coords", "k_coords", "lse", "workspace")] + \
               [("workspace_bytes", C.c_uint64)]


class vpe_block_norm_args(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "rows", "dim", "requests", "post", "pre")] + [("residual_scale", C.c_float), ("eps", C.c_float)] + \
               [(n, C.c_void_p) for n in ("x", "branch", "out", "normed")] + [(n, C.c_int64) for n in ("x_row", "branch_row", "out_row", "normed_row")] + \
               [(n, C.c_void_p) for n in ("post_gain", "post_bias", "pre_gain", "pre_bias", "layer_scale", "gate", "scale", "shift", "request")]


class vpe_adapter_linear_args(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "out_f32", "rows", "in_features", "out_features", "adapters", "rank")] + \
               [(n, C.c_void_p) for n in ("x", "weight", "bias", "out")] + [(n, C.c_int64) for n in ("x_row", "out_row")] + \
               [(n, C.c_void_p) for n in ("a", "b", "adapter", "scale", "workspace")] + [("workspace_bytes", C.c_uint64)]


class VpeError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"vpe error {code}: {msg}")
        self.code = code


def load_library(path: Optional[str] = None):
    """Load libvpe.so (building it first if it has never been built)."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or _LIB_PATH
    if not os.path.exists(p):
        from .build import build
        build()
    L = C.CDLL(p)
    vp, i32, i64p = C.c_void_p, C.c_int, C.POINTER(C.c_int64)
    L.vpe_workspace_bytes.argtypes = [C.POINTER(vpe_backbone_cfg), C.POINTER(vpe_head_cfg), i32, C.POINTER(C.c_uint64)]
    L.vpe_create.argtypes = [C.POINTER(vpe_backbone_cfg), C.POINTER(vpe_head_cfg), i32, vp, C.c_uint64, C.POINTER(vp)]
    L.vpe_encode.argtypes = [vp, vp, vp, C.POINTER(vpe_feat)]
    L.vpe_run_head.argtypes = [vp, i32, vpe_feat, vp]
    L.vpe_run_head_static.argtypes = [vp, i32, vpe_feat, vp]
    L.vpe_run_head_latest.argtypes = [vp, i32, vp, C.POINTER(vpe_feat)]
    L.vpe_head_counters.argtypes = [vp, i32, i64p]
    L.vpe_frame_ready.argtypes = [vp, vpe_feat]
    L.vpe_set_head_rate.argtypes = [vp, i32, i32]
    L.vpe_next_encode_stream.argtypes = [vp, C.POINTER(C.c_void_p)]
    L.vpe_preprocess_u8.argtypes = [vp, i32, i32, i32, vp, i32, i32, C.POINTER(C.c_float), C.POINTER(C.c_float), vp]
    L.vpe_encode_at.argtypes = [vp, vp, vp, C.c_double, C.POINTER(vpe_feat)]
    L.vpe_set_head_rate_hz.argtypes = [vp, i32, C.c_double]
    L.vpe_feat_view.argtypes = [vp, vpe_feat, i32, C.POINTER(vp), i64p]
    L.vpe_set_head_adapters.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp]
    L.vpe_head_output.argtypes = [vp, i32, i32, C.POINTER(vp), i64p]
    L.vpe_sync.argtypes = [vp]
    L.vpe_head_done.argtypes = [vp, i32]
    L.vpe_wait_head.argtypes = [vp, i32]
    L.vpe_stage_times.argtypes = [vp, C.POINTER(C.c_float), C.POINTER(C.c_float), i32]
    L.vpe_stats.argtypes = [vp, i64p, i64p, i64p, i32]
    L.vpe_time_kernel.argtypes = [vp, i32, i32, C.POINTER(C.c_float), C.POINTER(C.c_double), C.POINTER(C.c_double)]
    L.vpe_attention_workspace_bytes.argtypes = [C.POINTER(vpe_attention_args), C.POINTER(C.c_uint64)]
    L.vpe_attention.argtypes = [vp, vp]              # (a struct by reference, or its packed bytes)
    L.vpe_block_norm.argtypes = [vp, vp]              # (a struct by reference, or its packed bytes)
    L.vpe_adapter_linear_workspace_bytes.argtypes = [C.POINTER(vpe_adapter_linear_args), C.POINTER(C.c_uint64)]
    L.vpe_adapter_linear.argtypes = [vp, vp]              # (a struct by reference, or its packed bytes)
    L.vpe_last_error.argtypes = [vp]
    L.vpe_last_error.restype = C.c_char_p
    L.vpe_destroy.argtypes = [vp]
    L.vpe_destroy.restype = None
    for n in ("vpe_workspace_bytes", "vpe_create", "vpe_encode", "vpe_encode_at", "vpe_run_head", "vpe_set_head_rate", "vpe_set_head_adapters",
              "vpe_set_head_rate_hz", "vpe_preprocess_u8", "vpe_attention_workspace_bytes", "vpe_attention", "vpe_block_norm",
              "vpe_adapter_linear_workspace_bytes", "vpe_adapter_linear", "vpe_next_encode_stream", "vpe_feat_view",
              "vpe_head_output", "vpe_sync", "vpe_run_head_static", "vpe_head_done", "vpe_wait_head", "vpe_stage_times", "vpe_stats", "vpe_time_kernel", "vpe_run_head_latest", "vpe_head_counters", "vpe_frame_ready"):
        getattr(L, n).restype = C.c_int
    if path is None:
        _lib = L
    return L


def lib():
    return load_library()


# ------------------------------------------------------------------ the C calls, same names
def vpe_last_error(engine=None) -> str:
    return (lib().vpe_last_error(engine) or b"").decode()


def vpe_workspace_bytes(cfg: vpe_backbone_cfg, heads, n_heads: int) -> int:
    out = C.c_uint64(0)
    rc = lib().vpe_workspace_bytes(C.byref(cfg), heads, n_heads, C.byref(out))
    if rc:
        raise VpeError(rc, vpe_last_error())
    return int(out.value)


def vpe_create(cfg: vpe_backbone_cfg, heads, n_heads: int, workspace_ptr: Optional[int], workspace_bytes: int):
    out = C.c_void_p()
    rc = lib().vpe_create(C.byref(cfg), heads, n_heads, workspace_ptr, workspace_bytes, C.byref(out))
    if rc:
        raise VpeError(rc, vpe_last_error())
    return out


def vpe_encode(engine, images_ptr: int, stream_ptr: Optional[int] = None) -> vpe_feat:
    fh = vpe_feat()
    rc = lib().vpe_encode(engine, images_ptr, stream_ptr, C.byref(fh))
    if rc:
        raise VpeError(rc, vpe_last_error(engine))
    return fh


def vpe_preprocess_u8(frames_ptr: int, batch: int, src_h: int, src_w: int, images_ptr: int, dst_h: int, dst_w: int,
                      mean, std, stream_ptr: Optional[int] = None) -> None:
    m = (C.c_float * 3)(*[float(v) for v in mean])
    s = (C.c_float * 3)(*[float(v) for v in std])
    rc = lib().vpe_preprocess_u8(frames_ptr, batch, src_h, src_w, images_ptr, dst_h, dst_w, m, s, stream_ptr)
    if rc:
        raise VpeError(rc, vpe_last_error(None))


def preprocess_u8(frames, out, mean, std, stream=None) -> None:
    """frames: torch uint8 CUDA tensor [B, Hs, Ws, 3]; out: torch float32 CUDA tensor [B, 3, H, W] (written).
    stream: a torch stream, a raw hipStream_t as int (e.g. Engine.next_encode_stream()), or None."""
    assert frames.is_cuda and frames.is_contiguous() and frames.element_size() == 1 and frames.dim() == 4 and frames.shape[3] == 3
    assert out.is_cuda and out.is_contiguous() and out.dtype.is_floating_point and out.element_size() == 4
    assert out.dim() == 4 and out.shape[0] == frames.shape[0] and out.shape[1] == 3
    vpe_preprocess_u8(frames.data_ptr(), frames.shape[0], frames.shape[1], frames.shape[2], out.data_ptr(),
                      out.shape[2], out.shape[3], mean, std,
                      None if stream is None else stream if isinstance(stream, int) else stream.cuda_stream)


# ------------------------------------------------------------------ operators on packed rows
# A call takes some microseconds on the device: its arguments are packed in one go (the layouts are those of the structs above) and the
# tensors are looked at as little as the checks allow.
_PACK_ATTENTION = Struct("10i2f4Q8q9QQ")
_PACK_BLOCK_NORM = Struct("6i2f4Q4q9Q")
_PACK_ADAPTER = Struct("7i4x4Q2q5QQ")
assert (_PACK_ATTENTION.size, _PACK_BLOCK_NORM.size, _PACK_ADAPTER.size) == tuple(
    C.sizeof(t) for t in (vpe_attention_args, vpe_block_norm_args, vpe_adapter_linear_args))


def _refuse(message: str):
    raise VpeError(VPE_EINVAL, message)


def _types():
    """torch and its type objects, once torch is wanted."""
    global _torch, _f32, _bf16, _i32, _u8
    if _torch is None:
        import torch
        _f32, _bf16, _i32, _u8, _torch = torch.float32, torch.bfloat16, torch.int32, torch.uint8, torch
    return _torch


_torch = _f32 = _bf16 = _i32 = _u8 = None


def _dtype_of(t) -> int:
    d = t.dtype
    if d is _bf16:
        return VPE_BF16
    if d is _f32:
        return VPE_F32
    _refuse(f"tensors must be bfloat16 or float32, not {d}")


def _ptr(name: str, t, index: int, dtype, shape) -> int:
    """The address of a contiguous tensor that a call is to use, 0 for None; what does not fit is refused."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != index:
        _refuse(f"{name}: contiguous {dtype} {tuple(shape)} on device {index} expected, not {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _workspace(t, index: int):
    if t is None:
        return 0, 0
    if t.dtype is not _u8 or not t.is_contiguous() or t.get_device() != index:
        _refuse("workspace must be a contiguous uint8 tensor on the tensors' device")
    return t.data_ptr(), t.numel()


def _pack(form, *values) -> bytes:
    try:
        return form.pack(*values)
    except (StructError, OverflowError) as e:             # (a size that is no integer of its field's width)
        _refuse(str(e))


def _enqueue(call, packed: bytes, index: int, stream) -> None:
    """Makes the call with the tensors' device current; stream: a torch stream, a raw hipStream_t as int, or None (the default stream)."""
    if index < 0:
        _refuse("tensors must be in device memory")
    raw = None if stream is None else stream if isinstance(stream, int) else stream.cuda_stream
    if _torch.cuda.current_device() == index:
        rc = call(packed, raw)
    else:
        with _torch.cuda.device(index):
            rc = call(packed, raw)
    if rc:
        raise VpeError(rc, vpe_last_error(None))


def _row_stride(name: str, t) -> int:
    rows, cols = t.shape
    stride = t.stride()
    if cols > 1 and stride[1] != 1:
        _refuse(f"{name} must be a matrix with contiguous rows")
    return stride[0] if rows > 1 else max(stride[0], cols)            # (the stride of a single row says nothing)


def _attention_sizes(q, k):
    _types()
    if q.dim() != 3 or k.dim() != 3 or q.dtype is not k.dtype:
        _refuse("q and k must be [rows, heads, head_dim] of one type")
    (q_rows, heads, head_dim), (k_rows, kv_heads, k_dim) = q.shape, k.shape
    if head_dim != k_dim:
        _refuse("q and k must have the same head_dim")
    return _dtype_of(q), q_rows, heads, head_dim, k_rows, kv_heads


def attention_workspace_bytes(q, k, *, sequences: int, max_q: int, max_k: int) -> int:
    """Bytes of workspace that `attention` needs for tensors of these shapes, whatever the offsets say."""
    a, out = vpe_attention_args(), C.c_uint64(0)
    a.dtype, a.q_rows, a.heads, a.head_dim, a.k_rows, a.kv_heads = _attention_sizes(q, k)
    a.sequences, a.max_q, a.max_k = sequences, max_q, max_k
    rc = lib().vpe_attention_workspace_bytes(C.byref(a), C.byref(out))
    if rc:
        raise VpeError(rc, vpe_last_error(None))
    return int(out.value)


def _heads_matrix(name: str, t, shape, dtype, index: int):
    """(address, stride of the rows, of the heads) of a [rows, heads, head_dim] tensor."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != index:
        _refuse(f"{name}: {dtype} {tuple(shape)} on device {index} expected, not {t.dtype} {tuple(t.shape)} on {t.device}")
    row, head, last = t.stride()
    rows, heads, dim = shape
    if last != 1 and rows:
        _refuse(f"{name}'s last axis must be contiguous")
    return t.data_ptr(), row if rows > 1 else heads * dim, head if heads > 1 else dim       # (the stride of an axis of length one says nothing)


def attention(q, k, v, out, *, q_offsets, k_offsets, max_q: int, max_k: int, k_lengths=None, causal: bool = False, prefix=None,
              scale: Optional[float] = None, cap: float = 0.0, slopes=None, q_coords=None, k_coords=None, lse=None, workspace=None,
              stream=None) -> None:
    """vpe_attention on torch CUDA tensors: q, out [q_rows, heads, head_dim], k, v [k_rows, kv_heads, head_dim] (rows and heads of any
    stride, last axis contiguous; bfloat16 or float32); q_offsets, k_offsets int32 [sequences + 1], k_lengths, prefix int32
    [sequences]; slopes float32 [heads]; coordinates float32 [rows, 2]; lse float32 [q_rows, heads] (written, as is out).
    scale: 1 / sqrt(head_dim) if not given.  workspace: a uint8 tensor of attention_workspace_bytes.  stream: a torch stream, a raw
    hipStream_t as int, or None (the default stream)."""
    dtype, q_rows, heads, head_dim, k_rows, kv_heads = _attention_sizes(q, k)
    dev, sequences, q_shape, k_shape = q.get_device(), q_offsets.numel() - 1, q.shape, k.shape
    qp, q_row, q_head = _heads_matrix("q", q, q_shape, q.dtype, dev)
    kp, k_row, k_head = _heads_matrix("k", k, k_shape, q.dtype, dev)
    vp, v_row, v_head = _heads_matrix("v", v, k_shape, q.dtype, dev)
    op, o_row, o_head = _heads_matrix("out", out, q_shape, q.dtype, dev)
    ends, each = (sequences + 1,), (sequences,)
    wp, wb = _workspace(workspace, dev)
    packed = _pack(
        _PACK_ATTENTION, dtype, heads, kv_heads, head_dim, sequences, max_q, max_k, q_rows, k_rows, 1 if causal else 0, head_dim ** -0.5 if scale is None else scale, cap,
        qp, kp, vp, op, q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head, _ptr("q_offsets", q_offsets, dev, _i32, ends),
        _ptr("k_offsets", k_offsets, dev, _i32, ends), _ptr("k_lengths", k_lengths, dev, _i32, each), _ptr("prefix", prefix, dev, _i32, each),
        _ptr("slopes", slopes, dev, _f32, (heads,)), _ptr("q_coords", q_coords, dev, _f32, (q_rows, 2)),
        _ptr("k_coords", k_coords, dev, _f32, (k_rows, 2)), _ptr("lse", lse, dev, _f32, (q_rows, heads)), wp, wb)
    _enqueue(lib().vpe_attention, packed, dev, stream)


def _matrix(name: str, t, shape, dtype, index: int):
    """(address, stride of the rows) of a matrix whose rows may be strided, zeros for None."""
    if t is None:
        return 0, 0
    if t.dtype is not dtype or t.shape != shape or t.get_device() != index:
        _refuse(f"{name}: {dtype} {tuple(shape)} on device {index} expected, not {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr(), _row_stride(name, t)


def block_norm(x, out, *, branch=None, normed=None, post: int = VPE_NORM_NONE, post_gain=None, post_bias=None, pre: int = VPE_NORM_NONE,
               pre_gain=None, pre_bias=None, layer_scale=None, residual_scale: float = 1.0, gate=None, scale=None, shift=None,
               request=None, eps: float = 1e-6, stream=None) -> None:
    """vpe_block_norm on torch CUDA tensors: x, out float32 [rows, dim] (out is written and may be x); branch, normed [rows, dim],
    bfloat16 or float32 (normed is written); gains, biases and layer_scale float32 [dim]; gate, scale, shift float32 [requests, dim];
    request int32 [rows].  Rows may be strided.  stream: as for attention."""
    _types()
    if x.dim() != 2:
        _refuse("x must be a matrix")
    shape, dev = x.shape, x.get_device()
    rows, dim = shape
    typed = branch if branch is not None else normed
    dtype, t = (VPE_F32, _f32) if typed is None else (_dtype_of(typed), typed.dtype)
    xp, x_row = _matrix("x", x, shape, _f32, dev)
    op, out_row = _matrix("out", out, shape, _f32, dev)
    bp, branch_row = _matrix("branch", branch, shape, t, dev)
    np_, normed_row = _matrix("normed", normed, shape, t, dev)
    table = gate if gate is not None else scale if scale is not None else shift
    requests = 0 if table is None else table.shape[0]
    vector, modulation = (dim,), (requests, dim)
    packed = _pack(
        _PACK_BLOCK_NORM, dtype, rows, dim, requests, post, pre, residual_scale, eps, xp, bp, op, np_, x_row, branch_row, out_row, normed_row,
        _ptr("post_gain", post_gain, dev, _f32, vector), _ptr("post_bias", post_bias, dev, _f32, vector), _ptr("pre_gain", pre_gain, dev, _f32, vector),
        _ptr("pre_bias", pre_bias, dev, _f32, vector), _ptr("layer_scale", layer_scale, dev, _f32, vector), _ptr("gate", gate, dev, _f32, modulation),
        _ptr("scale", scale, dev, _f32, modulation), _ptr("shift", shift, dev, _f32, modulation), _ptr("request", request, dev, _i32, (rows,)))
    _enqueue(lib().vpe_block_norm, packed, dev, stream)


def _adapter_sizes(x, weight, a):
    _types()
    if x.dim() != 2 or weight.dim() != 2 or x.dtype is not weight.dtype:
        _refuse("x must be [rows, in_features], weight [out_features, in_features] of one type")
    (rows, in_features), (out_features, columns) = x.shape, weight.shape
    if in_features != columns:
        _refuse("weight must be [out_features, in_features]")
    if a is None:
        return _dtype_of(x), rows, in_features, out_features, 0, 0
    if a.dim() != 3 or a.shape[2] != in_features:
        _refuse("a must be [adapters, rank, in_features]")
    return _dtype_of(x), rows, in_features, out_features, a.shape[0], a.shape[1]


def adapter_linear_workspace_bytes(x, weight, a=None) -> int:
    """Bytes of workspace that `adapter_linear` needs for tensors of these shapes."""
    p, out = vpe_adapter_linear_args(), C.c_uint64(0)
    p.dtype, p.rows, p.in_features, p.out_features, p.adapters, p.rank = _adapter_sizes(x, weight, a)
    rc = lib().vpe_adapter_linear_workspace_bytes(C.byref(p), C.byref(out))
    if rc:
        raise VpeError(rc, vpe_last_error(None))
    return int(out.value)


def adapter_linear(x, weight, out, *, bias=None, a=None, b=None, adapter=None, scale=None, workspace=None, stream=None) -> None:
    """vpe_adapter_linear on torch CUDA tensors: x [rows, in_features] (rows may be strided), weight [out_features, in_features],
    a [adapters, rank, in_features], b [adapters, out_features, rank], all bfloat16 or all float32; out [rows, out_features] of
    that type or float32 (written); bias float32 [out_features]; adapter int32 [rows] (outside 0 .. adapters - 1: none); scale float32
    [adapters].  workspace: a uint8 tensor of adapter_linear_workspace_bytes.  stream: as for attention."""
    dtype, rows, in_features, out_features, adapters, rank = _adapter_sizes(x, weight, a)
    if (a is None) != (b is None) or (a is None) != (adapter is None):
        _refuse("a, b and adapter go together")
    dev, t = x.get_device(), x.dtype
    out_f32 = out.dtype is _f32
    xp, x_row = _matrix("x", x, x.shape, t, dev)
    op, out_row = _matrix("out", out, (rows, out_features), _f32 if out_f32 else t, dev)
    wp, wb = _workspace(workspace, dev)
    packed = _pack(
        _PACK_ADAPTER, dtype, 1 if out_f32 else 0, rows, in_features, out_features, adapters, rank, xp, _ptr("weight", weight, dev, t, weight.shape),
        _ptr("bias", bias, dev, _f32, (out_features,)), op, x_row, out_row, _ptr("a", a, dev, t, (adapters, rank, in_features)),
        _ptr("b", b, dev, t, (adapters, out_features, rank)), _ptr("adapter", adapter, dev, _i32, (rows,)), _ptr("scale", scale, dev, _f32, (adapters,)), wp, wb)
    _enqueue(lib().vpe_adapter_linear, packed, dev, stream)


def vpe_next_encode_stream(engine) -> Optional[int]:
    out = C.c_void_p()
    rc = lib().vpe_next_encode_stream(engine, C.byref(out))
    if rc:
        raise VpeError(rc, vpe_last_error(engine))
    return out.value


def vpe_encode_at(engine, images_ptr: int, stream_ptr: Optional[int], t_seconds: float) -> vpe_feat:
    fh = vpe_feat()
    rc = lib().vpe_encode_at(engine, images_ptr, stream_ptr, t_seconds, C.byref(fh))
    if rc:
        raise VpeError(rc, vpe_last_error(engine))
    return fh


def vpe_run_head(engine, head: int, fh: vpe_feat, stream_ptr: Optional[int] = None) -> int:
    rc = lib().vpe_run_head(engine, head, fh, stream_ptr)
    if rc < 0:
        raise VpeError(rc, vpe_last_error(engine))
    return rc


def vpe_run_head_static(engine, head: int, fh: vpe_feat, stream_ptr: Optional[int] = None) -> int:
    rc = lib().vpe_run_head_static(engine, head, fh, stream_ptr)
    if rc < 0:
        raise VpeError(rc, vpe_last_error(engine))
    return rc


def vpe_run_head_latest(engine, head: int, stream_ptr: Optional[int] = None):
    """Returns (status, handle): handle is the frame the head was started on, None unless status == VPE_OK."""
    fh = vpe_feat()
    rc = lib().vpe_run_head_latest(engine, head, stream_ptr, C.byref(fh))
    if rc < 0:
        raise VpeError(rc, vpe_last_error(engine))
    return rc, (fh if rc == VPE_OK else None)


def vpe_frame_ready(engine, fh: vpe_feat) -> int:
    """VPE_OK, VPE_BUSY or VPE_ESTALE."""
    rc = lib().vpe_frame_ready(engine, fh)
    if rc < 0 and rc != VPE_ESTALE:
        raise VpeError(rc, vpe_last_error(engine))
    return rc


HEAD_COUNTERS = ("runs", "skips", "missed", "overflow", "busy", "last_run_frame", "seen")


def vpe_head_counters(engine, head: int) -> dict:
    out = (C.c_int64 * 8)()
    rc = lib().vpe_head_counters(engine, head, out)
    if rc:
        raise VpeError(rc, vpe_last_error(engine))
    return {k: int(out[i]) for i, k in enumerate(HEAD_COUNTERS)}


def vpe_set_head_rate(engine, head: int, every_n_frames: int) -> None:
    rc = lib().vpe_set_head_rate(engine, head, every_n_frames)
    if rc:
        raise VpeError(rc, vpe_last_error(engine))


def vpe_set_head_rate_hz(engine, head: int, max_hz: float) -> None:
    rc = lib().vpe_set_head_rate_hz(engine, head, max_hz)
    if rc:
        raise VpeError(rc, vpe_last_error(engine))


def vpe_set_head_adapters(engine, head: int, adapters: int, rank: int, a_ptr, b_ptr, scale_ptr, adapter_of_image: Sequence[int]) -> None:
    rc = lib().vpe_set_head_adapters(engine, head, adapters, rank, a_ptr, b_ptr, scale_ptr,
                                     (C.c_int32 * len(adapter_of_image))(*adapter_of_image) if adapters else None)
    if rc:
        raise VpeError(rc, vpe_last_error(engine))


def vpe_feat_view(engine, fh: vpe_feat, tap: int):
    ptr = C.c_void_p()
    shape = (C.c_int64 * 3)()
    rc = lib().vpe_feat_view(engine, fh, tap, C.byref(ptr), shape)
    if rc:
        raise VpeError(rc, vpe_last_error(engine))
    return ptr.value, tuple(shape)


def vpe_head_output(engine, head: int, which: int):
    ptr = C.c_void_p()
    shape = (C.c_int64 * 4)()
    rc = lib().vpe_head_output(engine, head, which, C.byref(ptr), shape)
    if rc:
        raise VpeError(rc, vpe_last_error(engine))
    return ptr.value, tuple(shape)


def vpe_sync(engine) -> None:
    rc = lib().vpe_sync(engine)
    if rc:
        raise VpeError(rc, vpe_last_error(engine))


def vpe_head_done(engine, head: int) -> int:
    """VPE_OK or VPE_BUSY."""
    rc = lib().vpe_head_done(engine, head)
    if rc < 0:
        raise VpeError(rc, vpe_last_error(engine))
    return rc


def vpe_wait_head(engine, head: int) -> None:
    rc = lib().vpe_wait_head(engine, head)
    if rc:
        raise VpeError(rc, vpe_last_error(engine))


def vpe_stage_times(engine, n_heads: int):
    """(encode_ms, [head_ms...]); -1 where there is no figure yet."""
    enc = C.c_float(-1.0)
    heads = (C.c_float * max(n_heads, 1))()
    rc = lib().vpe_stage_times(engine, C.byref(enc), heads, n_heads)
    if rc:
        raise VpeError(rc, vpe_last_error(engine))
    return float(enc.value), [float(v) for v in heads][:n_heads]


def vpe_stats(engine, n_heads: int):
    frames = C.c_int64(0)
    runs = (C.c_int64 * max(n_heads, 1))()
    skips = (C.c_int64 * max(n_heads, 1))()
    lib().vpe_stats(engine, C.byref(frames), runs, skips, n_heads)
    return int(frames.value), [int(v) for v in runs][:n_heads], [int(v) for v in skips][:n_heads]


def vpe_time_kernel(engine, which: int, reps: int):
    ms, fl, by = C.c_float(0), C.c_double(0), C.c_double(0)
    rc = lib().vpe_time_kernel(engine, which, reps, C.byref(ms), C.byref(fl), C.byref(by))
    if rc:
        raise VpeError(rc, vpe_last_error(engine))
    return float(ms.value), float(fl.value), float(by.value)


def vpe_destroy(engine) -> None:
    lib().vpe_destroy(engine)


# ------------------------------------------------------------------ convenience wrapper
@dataclass
class HeadCfg:
    kind: int
    weights: np.ndarray        # flat fp32 blob in the documented order
    classes: int = 0
    channels: int = 0
    every_n: int = 1


class Engine:
    """Owns one vpe_engine.  Device memory comes from torch (one uint8 tensor), streams are
    the library's own unless torch streams are passed in."""

    def __init__(self, *, dim, depth, heads, mlp_hidden, img_h, img_w, weights: np.ndarray, taps,
                 mlp_kind=VPE_MLP_GELU, registers=0, batch=1, dtype=VPE_BF16, ring_slots=2, flags=0, ln_eps=1e-6,
                 encoder_lanes=1, head_streams=0,
                 head_cfgs: Sequence[HeadCfg] = (), torch_workspace: bool = True):
        self._keep = [np.ascontiguousarray(weights, dtype=np.float32)]
        cfg = vpe_backbone_cfg()
        cfg.dim, cfg.depth, cfg.heads, cfg.mlp_hidden, cfg.mlp_kind = dim, depth, heads, mlp_hidden, mlp_kind
        cfg.registers, cfg.img_h, cfg.img_w, cfg.batch, cfg.dtype = registers, img_h, img_w, batch, dtype
        cfg.taps = (C.c_int32 * 4)(*taps)
        cfg.ring_slots, cfg.flags, cfg.ln_eps, cfg.encoder_lanes = ring_slots, flags, ln_eps, encoder_lanes
        cfg.head_streams = head_streams
        cfg.weights = self._keep[0].ctypes.data
        cfg.weights_bytes = self._keep[0].nbytes
        self.n_heads = len(head_cfgs)
        harr = (vpe_head_cfg * max(self.n_heads, 1))()
        for i, h in enumerate(head_cfgs):
            blob = np.ascontiguousarray(h.weights, dtype=np.float32)
            self._keep.append(blob)
            harr[i].kind, harr[i].classes, harr[i].channels, harr[i].every_n = h.kind, h.classes, h.channels, h.every_n
            harr[i].weights = blob.ctypes.data
            harr[i].weights_bytes = blob.nbytes
        self.cfg, self.head_arr = cfg, harr
        self.host_only = bool(flags & VPE_FLAG_HOST_ONLY)
        self._adapters = {}                       # head -> the tensors that its runs read
        self.dtype = dtype
        self.workspace_bytes = vpe_workspace_bytes(cfg, harr, self.n_heads)
        self._ws = None
        ws_ptr, ws_bytes = None, 0
        if torch_workspace and not self.host_only:
            import torch
            self._ws = torch.empty(self.workspace_bytes + 256, dtype=torch.uint8, device="cuda")
            ws_ptr = (self._ws.data_ptr() + 255) // 256 * 256
            ws_bytes = self.workspace_bytes
        self.handle = vpe_create(cfg, harr, self.n_heads, ws_ptr, ws_bytes)

    # -- calls
    def encode(self, images, stream=None, t: Optional[float] = None) -> vpe_feat:
        """images: torch float32 CUDA tensor [B,3,H,W] (contiguous) -- or None in host-only mode.
        t: capture time of the frame in seconds (for per-head limits in Hz), or None."""
        ptr = sp = None
        if not self.host_only:
            assert images.is_cuda and images.is_contiguous() and images.dtype.is_floating_point and images.element_size() == 4
            assert tuple(images.shape) == (self.cfg.batch, 3, self.cfg.img_h, self.cfg.img_w), images.shape
            ptr, sp = images.data_ptr(), None if stream is None else stream.cuda_stream
        return vpe_encode(self.handle, ptr, sp) if t is None else vpe_encode_at(self.handle, ptr, sp, t)

    def run_head(self, head: int, fh: vpe_feat, stream=None) -> int:
        return vpe_run_head(self.handle, head, fh, None if stream is None else stream.cuda_stream)

    def run_head_static(self, head: int, fh: vpe_feat, stream=None) -> int:
        return vpe_run_head_static(self.handle, head, fh, None if stream is None else stream.cuda_stream)

    def run_head_latest(self, head: int, stream=None):
        return vpe_run_head_latest(self.handle, head, None if stream is None else stream.cuda_stream)

    def frame_ready(self, fh: vpe_feat) -> int:
        return vpe_frame_ready(self.handle, fh)

    def head_counters(self, head: int) -> dict:
        return vpe_head_counters(self.handle, head)

    def next_encode_stream(self) -> Optional[int]:
        """Raw handle of the engine stream the next encode() without a stream argument will run on."""
        return vpe_next_encode_stream(self.handle)

    def set_head_rate(self, head: int, every_n: int) -> None:
        vpe_set_head_rate(self.handle, head, every_n)

    def set_head_rate_hz(self, head: int, max_hz: float) -> None:
        vpe_set_head_rate_hz(self.handle, head, max_hz)

    def set_head_adapters(self, head: int, a=None, b=None, adapter_of_image: Sequence[int] = (), scale=None) -> None:
        """Adapters of a query head's kv projection: a [adapters, rank, dim], b [adapters, 2 dim, rank] in the engine's dtype, scale float32
        [adapters]; adapter_of_image [batch], -1 for none.  Kept by the engine until the next call; without arguments they are taken away."""
        if a is None:
            vpe_set_head_adapters(self.handle, head, 0, 0, None, None, None, ())
        else:
            _types()
            dtype, dim = _bf16 if self.dtype == VPE_BF16 else _f32, self.cfg.dim
            if a.dim() != 3 or len(adapter_of_image) != self.cfg.batch:
                _refuse("a must be [adapters, rank, dim], adapter_of_image one index an image")
            if a.get_device() < 0 and not self.host_only:
                _refuse("tensors must be in device memory")
            n, rank, device = a.shape[0], a.shape[1], self._ws.get_device() if self._ws is not None else a.get_device()
            ptrs = (_ptr("a", a, device, dtype, (n, rank, dim)), _ptr("b", b, device, dtype, (n, 2 * dim, rank)), _ptr("scale", scale, device, _f32, (n,)))
            vpe_set_head_adapters(self.handle, head, n, rank, *ptrs, [i if 0 <= i < n else -1 for i in adapter_of_image])
        self._adapters[head] = (a, b, scale)

    def sync(self) -> None:
        vpe_sync(self.handle)

    def stats(self):
        return vpe_stats(self.handle, self.n_heads)

    def head_done(self, head: int) -> bool:
        return vpe_head_done(self.handle, head) == VPE_OK

    def wait_head(self, head: int) -> None:
        vpe_wait_head(self.handle, head)

    def stage_times(self):
        return vpe_stage_times(self.handle, self.n_heads)

    def time_kernel(self, which: int, reps: int):
        return vpe_time_kernel(self.handle, which, reps)

    # -- borrowed views as torch tensors (no copy)
    def _as_tensor(self, ptr: int, shape, torch_dtype):
        """Wrap library-owned device memory as a torch tensor (no copy, no ownership)."""
        import torch
        holder = _DevArray(ptr, tuple(int(s) for s in shape), torch_dtype)
        t = torch.as_tensor(holder, device="cuda")
        return t.view(torch.bfloat16) if torch_dtype == torch.bfloat16 else t

    def feat_view(self, fh: vpe_feat, tap: int):
        import torch
        ptr, shape = vpe_feat_view(self.handle, fh, tap)
        return self._as_tensor(ptr, shape, torch.bfloat16 if self.dtype == VPE_BF16 else torch.float32)

    def feat_ptr(self, fh: vpe_feat, tap: int) -> int:
        return vpe_feat_view(self.handle, fh, tap)[0]

    def head_output(self, head: int, which: int):
        import torch
        ptr, shape = vpe_head_output(self.handle, head, which)
        kind = self.head_arr[head].kind
        is_map = which == 1 and kind in (VPE_HEAD_SEG, VPE_HEAD_DET)
        shape = [s for s in shape]
        while len(shape) > 1 and shape[-1] == 1 and len(shape) > (3 if (is_map or kind in (VPE_HEAD_DEPTH, VPE_HEAD_DPT, VPE_HEAD_QUERY)) else 4):
            shape.pop()
        return self._as_tensor(ptr, shape, torch.uint8 if is_map else torch.float32)

    def close(self) -> None:
        if getattr(self, "handle", None):
            vpe_destroy(self.handle)
            self.handle = None
        self._ws = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class _DevArray:
    """Minimal __cuda_array_interface__ carrier so torch can wrap library-owned device memory."""
    _TYPESTR = {"torch.float32": "<f4", "torch.uint8": "|u1", "torch.bfloat16": "<i2"}

    def __init__(self, ptr: int, shape, torch_dtype):
        self.__cuda_array_interface__ = {"shape": shape, "typestr": self._TYPESTR[str(torch_dtype)],
                                         "data": (ptr, False), "version": 2, "strides": None}
