"""ctypes binding of the SAS C ABI (include/sas.h).

Argument marshalling only: every function here converts torch tensors to
device pointers, checks dtype/device/contiguity, and calls the entry point
of the same name in libsas.so.  No arithmetic of the method happens here, and
there is no fallback: if the library is missing or the device is not sm_103,
the calls raise.
"""
from __future__ import annotations

import collections
import contextlib
import ctypes
import os
import re

import torch

from . import _build

SAS_OK = 0
SAS_ERR_INVALID_ARG = 1
SAS_ERR_UNSUPPORTED = 2
SAS_ERR_CUDA = 3
SAS_ERR_TIMEOUT = 4
SAS_ERR_OOM = 5

SAS_MODE_TRAIN_SOFT = 0
SAS_MODE_INFER_HARD = 1
SAS_MODE_TRAIN_HARD_STE = 2
SAS_SEL_SCORES_GIVEN = 0
SAS_SEL_MEANPOOL_PROJ = 1
SAS_GATE_SOFTMAX = 0
SAS_GATE_SIGMOID = 1
SAS_GATE_LOGIT = 2
SAS_GATE_INNER = 0
SAS_GATE_OUTER = 1
SAS_SCOPE_SPARSE = 0
SAS_SCOPE_FULL = 1
SAS_NUM_KERNEL_KINDS = 8
KERNEL_KINDS = ["block_summaries", "query_projection", "selection", "attention", "mlp_up_gelu", "mlp_down",
                "attention_bwd", "qk_norm_rope"]

HEADER = os.path.join(_build.ROOT, "include", "sas.h")


class SasConfig(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("N", ctypes.c_int32), ("d", ctypes.c_int32),
                ("block", ctypes.c_int32), ("topk", ctypes.c_int32), ("sm_scale", ctypes.c_float),
                ("mode", ctypes.c_int32), ("selector", ctypes.c_int32), ("d_sel", ctypes.c_int32),
                ("gate_act", ctypes.c_int32), ("gate_pos", ctypes.c_int32), ("Hkv", ctypes.c_int32),
                ("max_seqs", ctypes.c_int32), ("max_seqlen", ctypes.c_int32), ("scope", ctypes.c_int32)]


class SasDecodeConfig(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("d", ctypes.c_int32),
                ("d_sel", ctypes.c_int32), ("block", ctypes.c_int32), ("topk", ctypes.c_int32),
                ("max_blocks", ctypes.c_int32), ("num_pages", ctypes.c_int32), ("sm_scale", ctypes.c_float),
                ("dense", ctypes.c_int32)]


class SasRopeConfig(ctypes.Structure):
    _fields_ = [("rot", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("max_pos", ctypes.c_int32),
                ("eps", ctypes.c_float)]


class SasChunkConfig(ctypes.Structure):
    _fields_ = [("max_seqs", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("d", ctypes.c_int32),
                ("block", ctypes.c_int32), ("max_blocks", ctypes.c_int32), ("num_pages", ctypes.c_int32),
                ("max_tokens", ctypes.c_int32), ("sm_scale", ctypes.c_float)]


SAS_DECODE_NUM_KERNEL_KINDS = 4
DECODE_KERNEL_KINDS = ["prep", "select", "attention", "summarize"]
SAS_CHUNK_NUM_KERNEL_KINDS = 4
CHUNK_KERNEL_KINDS = ["plan", "append", "attention", "verify"]


class SasError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"{message} (status {status})")
        self.status = status


_lib = None


def lib():
    """Loads libsas.so (built in-tree by _build.build())."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_build.LIB_PATH):
        raise RuntimeError("libsas.so is not built; run paper_2609_13141_gb300._build.build() first")
    L = ctypes.CDLL(_build.LIB_PATH)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    L.sas_create.argtypes = [ctypes.POINTER(SasConfig), ctypes.POINTER(vp)]
    L.sas_create.restype = i32
    L.sas_destroy.argtypes = [vp]
    L.sas_destroy.restype = None
    L.sas_attention_fwd.argtypes = [vp] * 12
    L.sas_attention_fwd.restype = i32
    L.sas_attention_fwd_noisy.argtypes = [vp] * 13
    L.sas_attention_fwd_noisy.restype = i32
    L.sas_attention_fwd_varlen.argtypes = [vp, vp, i32] + [vp] * 11
    L.sas_attention_fwd_varlen.restype = i32
    L.sas_attention_bwd.argtypes = [vp] * 16
    L.sas_attention_bwd.restype = i32
    L.sas_mlp_fwd.argtypes = [vp] * 7 + [i64, i64, i64, vp]
    L.sas_mlp_fwd.restype = i32
    L.sas_status_str.argtypes = [i32]
    L.sas_status_str.restype = ctypes.c_char_p
    L.sas_last_error.argtypes = [vp]
    L.sas_last_error.restype = ctypes.c_char_p
    L.sas_get_device_status.argtypes = [vp, ctypes.POINTER(i32)]
    L.sas_get_device_status.restype = i32
    L.sas_set_timing.argtypes = [vp, i32]
    L.sas_set_timing.restype = i32
    L.sas_get_timings.argtypes = [vp, ctypes.POINTER(i64), ctypes.POINTER(ctypes.c_double), i32]
    L.sas_get_timings.restype = i32
    L.sas_launch_count.argtypes = [vp]
    L.sas_launch_count.restype = i64
    L.sas_set_wait_limit.argtypes = [vp, i64]
    L.sas_set_wait_limit.restype = i32
    L.sas_get_tile_union_counts.argtypes = [vp, ctypes.POINTER(i32), i64]
    L.sas_get_tile_union_counts.restype = i32
    L.sas_get_attention_work.argtypes = [vp, ctypes.POINTER(i64), ctypes.POINTER(i64)]
    L.sas_get_attention_work.restype = i32
    L.sas_mlp_fwd_noalloc.argtypes = [vp] * 6 + [i64, i64, i64, vp]
    L.sas_mlp_fwd_noalloc.restype = i32
    L.sas_mlp_noalloc_get_device_status.argtypes = [ctypes.POINTER(i32)]
    L.sas_mlp_noalloc_get_device_status.restype = i32
    L.sas_selftest_wait_timeout.argtypes = [i64, ctypes.POINTER(i32)]
    L.sas_selftest_wait_timeout.restype = i32
    L.sas_decode_create.argtypes = [ctypes.POINTER(SasDecodeConfig), ctypes.POINTER(vp)]
    L.sas_decode_create.restype = i32
    L.sas_decode_destroy.argtypes = [vp]
    L.sas_decode_destroy.restype = None
    L.sas_decode_summarize.argtypes = [vp] * 7
    L.sas_decode_summarize.restype = i32
    L.sas_decode_step.argtypes = [vp] * 15
    L.sas_decode_step.restype = i32
    L.sas_decode_last_error.argtypes = [vp]
    L.sas_decode_last_error.restype = ctypes.c_char_p
    L.sas_decode_get_device_status.argtypes = [vp, ctypes.POINTER(i32)]
    L.sas_decode_get_device_status.restype = i32
    L.sas_decode_set_timing.argtypes = [vp, i32]
    L.sas_decode_set_timing.restype = i32
    L.sas_decode_get_timings.argtypes = [vp, ctypes.POINTER(i64), ctypes.POINTER(ctypes.c_double), i32]
    L.sas_decode_get_timings.restype = i32
    L.sas_decode_launch_count.argtypes = [vp]
    L.sas_decode_launch_count.restype = i64
    rope = ctypes.POINTER(SasRopeConfig)
    L.sas_qk_norm_rope_fwd.argtypes = [vp, rope, vp, i64] + [vp] * 9
    L.sas_qk_norm_rope_fwd.restype = i32
    L.sas_qk_norm_rope_bwd.argtypes = [vp, rope, vp, i64] + [vp] * 9 + [i64] + [vp] * 3
    L.sas_qk_norm_rope_bwd.restype = i32
    L.sas_chunk_create.argtypes = [ctypes.POINTER(SasChunkConfig), ctypes.POINTER(vp)]
    L.sas_chunk_create.restype = i32
    L.sas_chunk_destroy.argtypes = [vp]
    L.sas_chunk_destroy.restype = None
    L.sas_chunk_plan.argtypes = [vp, i32, i32, vp, vp, vp, vp, i32] + [vp] * 8
    L.sas_chunk_plan.restype = i32
    L.sas_chunk_append.argtypes = [vp, rope, i32, vp, i64] + [vp] * 10
    L.sas_chunk_append.restype = i32
    L.sas_chunk_attention.argtypes = [vp, i32, i32] + [vp] * 9
    L.sas_chunk_attention.restype = i32
    L.sas_chunk_verify.argtypes = [vp] + [i32] * 4 + [vp, vp, vp, i64, vp, i64, vp, vp, i64, vp, vp, vp]
    L.sas_chunk_verify.restype = i32
    L.sas_chunk_last_error.argtypes = [vp]
    L.sas_chunk_last_error.restype = ctypes.c_char_p
    L.sas_chunk_get_device_status.argtypes = [vp, ctypes.POINTER(i32)]
    L.sas_chunk_get_device_status.restype = i32
    L.sas_chunk_set_timing.argtypes = [vp, i32]
    L.sas_chunk_set_timing.restype = i32
    L.sas_chunk_get_timings.argtypes = [vp, ctypes.POINTER(i64), ctypes.POINTER(ctypes.c_double), i32]
    L.sas_chunk_get_timings.restype = i32
    L.sas_chunk_launch_count.argtypes = [vp]
    L.sas_chunk_launch_count.restype = i64
    L.sas_chunk_set_wait_limit.argtypes = [vp, i64]
    L.sas_chunk_set_wait_limit.restype = i32
    _lib = L
    return L


def header_functions():
    """Names of the functions include/sas.h declares."""
    text = open(HEADER).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(sas_[a-z_]+)\s*\(", text)))


def _ptr(t, dtype, name, required=True):
    if t is None:
        if required:
            raise ValueError(f"{name} is required")
        return None
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda":
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _arg(t, dtype, name, dev, shape=None):
    """Device address of a contiguous tensor on device `dev` (its index): like _ptr, with its shape and device checked,
    and a plain integer, for the entry points whose time is mostly the call's."""
    try:
        if t.dtype is dtype and t.get_device() == dev >= 0 and t.is_contiguous() and (shape is None or t.shape == shape):
            return t.data_ptr()
    except AttributeError:   # not a tensor
        pass
    _refuse(t, dtype, name, dev, shape)
    raise ValueError(f"{name} must be contiguous")


def _rows(t, dtype, name, dev, shape):
    """Device address of a tensor of any strides (its caller checks those)."""
    try:
        if t.dtype is dtype and t.get_device() == dev >= 0 and t.shape == shape:
            return t.data_ptr()
    except AttributeError:
        pass
    _refuse(t, dtype, name, dev, shape)


def _refuse(t, dtype, name, dev, shape):
    """Raises for what is wrong with a tensor argument, if it is not its strides."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.get_device() != dev:
        raise ValueError(f"{name} must be on device {dev}")


class _Handle(ctypes.c_void_p):
    """A handle with the sizes it was made with, which the tensors of its calls are compared with: the library takes
    addresses and goes by its own sizes."""
    sizes = None


def _sizes(h):
    sizes = getattr(h, "sizes", None)
    if sizes is None:
        raise SasError(SAS_ERR_INVALID_ARG, "the handle must be one that sas_create or sas_chunk_create returned, not closed")
    return sizes


def _rope_config(cos, eps, interleaved):
    try:
        max_pos, half = cos.shape
    except (AttributeError, ValueError):
        raise ValueError("cos must be a [max_pos, rot / 2] tensor") from None
    return SasRopeConfig(2 * half, 1 if interleaved else 0, max_pos, eps)


def _token_stride(t, name, lead):
    """Elements between two tokens of a [tokens.., heads, d] tensor (lead token axes): the heads of a token are
    contiguous, and all tokens evenly spaced."""
    st, sh = t.stride(), t.shape
    if (sh[-1] > 1 and st[-1] != 1) or (sh[-2] > 1 and st[-2] != sh[-1]):
        raise ValueError(f"{name}: the heads of a token must be contiguous")
    if lead == 1:
        return st[0] if sh[0] > 1 else sh[1] * sh[2]
    ld = st[1] if sh[1] > 1 else (st[0] if sh[0] > 1 else sh[2] * sh[3])
    if sh[0] > 1 and st[0] != sh[1] * ld:
        raise ValueError(f"{name}: the tokens of all batch rows must be evenly spaced")
    return ld


def _raw_stream(stream, dev):
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(dev)   # current_stream(dev).cuda_stream without the object
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


_HERE = contextlib.nullcontext()


def _on(stream):
    """Context in which outputs are allocated: the stream the call runs on, whose pool then owns them."""
    if stream is None:
        return _HERE
    if not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(int(stream))
    return torch.cuda.stream(stream)


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def _check(status, handle=None, what="sas"):
    if status != SAS_OK:
        L = lib()
        msg = L.sas_status_str(status).decode()
        if handle is not None:
            detail = L.sas_last_error(handle).decode()
            if detail:
                msg += ": " + detail
        raise SasError(status, f"{what}: {msg}")


def sas_status_str(status):
    return lib().sas_status_str(int(status)).decode()


def sas_create(B, H, N, d, topk, mode=SAS_MODE_TRAIN_SOFT, selector=SAS_SEL_SCORES_GIVEN, d_sel=0,
               sm_scale=0.0, block=64, gate_act=SAS_GATE_SOFTMAX, gate_pos=SAS_GATE_INNER, Hkv=0, max_seqs=0,
               max_seqlen=0, scope=SAS_SCOPE_SPARSE):
    cfg = SasConfig(B, H, N, d, block, topk, sm_scale, mode, selector, d_sel, gate_act, gate_pos, Hkv, max_seqs,
                    max_seqlen, scope)
    h = _Handle()
    _check(lib().sas_create(ctypes.byref(cfg), ctypes.byref(h)), None, "sas_create")
    h.sizes = B, H, Hkv or H, N, d
    return h


def sas_create_status(B, H, N, d, topk, mode=0, selector=0, d_sel=0, sm_scale=0.0, block=64,
                      gate_act=SAS_GATE_SOFTMAX, gate_pos=SAS_GATE_INNER, Hkv=0, max_seqs=0, max_seqlen=0,
                      scope=SAS_SCOPE_SPARSE):
    """Raw status of sas_create (for argument-check tests); destroys the handle on success."""
    cfg = SasConfig(B, H, N, d, block, topk, sm_scale, mode, selector, d_sel, gate_act, gate_pos, Hkv, max_seqs,
                    max_seqlen, scope)
    h = ctypes.c_void_p()
    st = lib().sas_create(ctypes.byref(cfg), ctypes.byref(h))
    if st == SAS_OK:
        lib().sas_destroy(h)
    return st


def sas_destroy(h):
    lib().sas_destroy(h)


def sas_attention_fwd_varlen(h, cu_seqlens, Q, K, V, scores, O, LSE=None, sel_idx=None, sel_logg=None,
                             stream=None, Wq=None, Wk=None):
    bf = torch.bfloat16
    st = lib().sas_attention_fwd_varlen(
        h, _ptr(cu_seqlens, torch.int32, "cu_seqlens"), ctypes.c_int32(cu_seqlens.numel() - 1),
        _ptr(Q, bf, "Q"), _ptr(K, bf, "K"), _ptr(V, bf, "V"), _ptr(scores, torch.float32, "scores", False),
        _ptr(Wq, bf, "Wq", False), _ptr(Wk, bf, "Wk", False), _ptr(O, bf, "O"), _ptr(LSE, torch.float32, "LSE", False), _ptr(sel_idx, torch.int32, "sel_idx", False),
        _ptr(sel_logg, torch.float32, "sel_logg", False), _stream(stream))
    _check(st, h, "sas_attention_fwd_varlen")


def sas_attention_fwd(h, Q, K, V, O, scores=None, Wq=None, Wk=None, LSE=None, sel_idx=None, sel_logg=None,
                      stream=None):
    bf = torch.bfloat16
    st = lib().sas_attention_fwd(
        h, _ptr(Q, bf, "Q"), _ptr(K, bf, "K"), _ptr(V, bf, "V"),
        _ptr(scores, torch.float32, "scores", False), _ptr(Wq, bf, "Wq", False), _ptr(Wk, bf, "Wk", False),
        _ptr(O, bf, "O"), _ptr(LSE, torch.float32, "LSE", False), _ptr(sel_idx, torch.int32, "sel_idx", False),
        _ptr(sel_logg, torch.float32, "sel_logg", False), _stream(stream))
    _check(st, h, "sas_attention_fwd")


def sas_attention_fwd_noisy(h, Q, K, V, O, noise, scores=None, Wq=None, Wk=None, LSE=None, sel_idx=None,
                            sel_logg=None, stream=None):
    bf = torch.bfloat16
    st = lib().sas_attention_fwd_noisy(
        h, _ptr(Q, bf, "Q"), _ptr(K, bf, "K"), _ptr(V, bf, "V"),
        _ptr(scores, torch.float32, "scores", False), _ptr(Wq, bf, "Wq", False), _ptr(Wk, bf, "Wk", False),
        _ptr(noise, torch.float32, "noise"), _ptr(O, bf, "O"), _ptr(LSE, torch.float32, "LSE", False),
        _ptr(sel_idx, torch.int32, "sel_idx", False), _ptr(sel_logg, torch.float32, "sel_logg", False),
        _stream(stream))
    _check(st, h, "sas_attention_fwd_noisy")


def sas_attention_bwd(h, Q, K, V, O, LSE, dO, dQ, dK, dV, scores=None, sel_idx=None, sel_logg=None, dlogg=None,
                      dscores=None, stream=None):
    bf, f32 = torch.bfloat16, torch.float32
    st = lib().sas_attention_bwd(
        h, _ptr(Q, bf, "Q"), _ptr(K, bf, "K"), _ptr(V, bf, "V"), _ptr(scores, f32, "scores", False),
        _ptr(O, bf, "O"), _ptr(LSE, f32, "LSE"), _ptr(dO, bf, "dO"), _ptr(sel_idx, torch.int32, "sel_idx", False),
        _ptr(sel_logg, f32, "sel_logg", False), _ptr(dQ, bf, "dQ"), _ptr(dK, bf, "dK"), _ptr(dV, bf, "dV"),
        _ptr(dlogg, f32, "dlogg", False), _ptr(dscores, f32, "dscores", False), _stream(stream))
    _check(st, h, "sas_attention_bwd")


def sas_qk_norm_rope_fwd(h, qkv, wq, wk, cos, sin, Q, K, V, positions=None, eps=1e-6, interleaved=False, stream=None):
    """qkv [B, N, H + 2 Hkv, d] (tokens evenly spaced, any distance) to Q [B, H, N, d], K and V [B, Hkv, N, d]."""
    B, H, Hkv, N, d = _sizes(h)
    dev, bf, f32 = Q.get_device(), torch.bfloat16, torch.float32
    cfg = _rope_config(cos, eps, interleaved)
    st = lib().sas_qk_norm_rope_fwd(
        h, cfg, _rows(qkv, bf, "qkv", dev, (B, N, H + 2 * Hkv, d)), _token_stride(qkv, "qkv", 2),
        _arg(wq, bf, "wq", dev, (d,)), _arg(wk, bf, "wk", dev, (d,)), _arg(cos, f32, "cos", dev), _arg(sin, f32, "sin", dev, cos.shape),
        None if positions is None else _arg(positions, torch.int32, "positions", dev, (B, N)), _arg(Q, bf, "Q", dev, (B, H, N, d)),
        _arg(K, bf, "K", dev, (B, Hkv, N, d)), _arg(V, bf, "V", dev, (B, Hkv, N, d)), _raw_stream(stream, dev))
    if st != SAS_OK:
        _check(st, h, "sas_qk_norm_rope_fwd")


def sas_qk_norm_rope_bwd(h, qkv, wq, wk, cos, sin, dQ, dK, dV, dqkv, dwq, dwk, positions=None, eps=1e-6,
                         interleaved=False, stream=None):
    """Gradients of sas_qk_norm_rope_fwd: dqkv like qkv, dwq and dwk fp32 [d]."""
    B, H, Hkv, N, d = _sizes(h)
    dev, bf, f32 = dQ.get_device(), torch.bfloat16, torch.float32
    rows = (B, N, H + 2 * Hkv, d)
    cfg = _rope_config(cos, eps, interleaved)
    st = lib().sas_qk_norm_rope_bwd(
        h, cfg, _rows(qkv, bf, "qkv", dev, rows), _token_stride(qkv, "qkv", 2), _arg(wq, bf, "wq", dev, (d,)),
        _arg(wk, bf, "wk", dev, (d,)), _arg(cos, f32, "cos", dev), _arg(sin, f32, "sin", dev, cos.shape),
        None if positions is None else _arg(positions, torch.int32, "positions", dev, (B, N)), _arg(dQ, bf, "dQ", dev, (B, H, N, d)),
        _arg(dK, bf, "dK", dev, (B, Hkv, N, d)), _arg(dV, bf, "dV", dev, (B, Hkv, N, d)), _rows(dqkv, bf, "dqkv", dev, rows),
        _token_stride(dqkv, "dqkv", 2), _arg(dwq, f32, "dwq", dev, (d,)), _arg(dwk, f32, "dwk", dev, (d,)),
        _raw_stream(stream, dev))
    if st != SAS_OK:
        _check(st, h, "sas_qk_norm_rope_bwd")


def sas_mlp_fwd(h, X, W1, W2, Y, b1=None, b2=None, stream=None):
    bf = torch.bfloat16
    T, D = X.shape
    F = W1.shape[0]
    st = lib().sas_mlp_fwd(h, _ptr(X, bf, "X"), _ptr(W1, bf, "W1"), _ptr(b1, bf, "b1", False), _ptr(W2, bf, "W2"),
                           _ptr(b2, bf, "b2", False), _ptr(Y, bf, "Y"), T, D, F, _stream(stream))
    _check(st, h, "sas_mlp_fwd")


SAS_MLP_NOALLOC_MAX_HIDDEN_BYTES = 32 * 1024 * 1024


def sas_mlp_fwd_noalloc(X, W1, W2, Y, b1=None, b2=None, stream=None):
    """The MLP without a handle and without any device allocation (see sas.h):
    the hidden activation lives in a fixed 32 MiB array inside the library,
    shared by every call on the device."""
    bf = torch.bfloat16
    T, D = X.shape
    F = W1.shape[0]
    st = lib().sas_mlp_fwd_noalloc(_ptr(X, bf, "X"), _ptr(W1, bf, "W1"), _ptr(b1, bf, "b1", False),
                                   _ptr(W2, bf, "W2"), _ptr(b2, bf, "b2", False), _ptr(Y, bf, "Y"), T, D, F,
                                   _stream(stream))
    if st == SAS_ERR_UNSUPPORTED and T * F * 2 > SAS_MLP_NOALLOC_MAX_HIDDEN_BYTES:
        raise SasError(st, f"sas_mlp_fwd_noalloc: hidden activation of {T}x{F} bf16 ({T * F * 2} bytes) exceeds "
                           f"the fixed {SAS_MLP_NOALLOC_MAX_HIDDEN_BYTES}-byte array")
    _check(st, None, "sas_mlp_fwd_noalloc")


def sas_mlp_noalloc_get_device_status():
    """Reads and clears the status word of sas_mlp_fwd_noalloc on the current
    device (synchronises the device)."""
    v = ctypes.c_int32(-1)
    _check(lib().sas_mlp_noalloc_get_device_status(ctypes.byref(v)), None, "sas_mlp_noalloc_get_device_status")
    return v.value


def sas_get_device_status(h):
    v = ctypes.c_int32(0)
    _check(lib().sas_get_device_status(h, ctypes.byref(v)), h, "sas_get_device_status")
    return v.value


def sas_set_timing(h, enable):
    _check(lib().sas_set_timing(h, 1 if enable else 0), h, "sas_set_timing")


def sas_get_timings(h):
    """{kind: (launches, total_ms)} for the kernel kinds of sas.h."""
    n = SAS_NUM_KERNEL_KINDS
    launches = (ctypes.c_int64 * n)()
    ms = (ctypes.c_double * n)()
    _check(lib().sas_get_timings(h, launches, ms, n), h, "sas_get_timings")
    return {KERNEL_KINDS[k]: (launches[k], ms[k]) for k in range(n)}


def sas_launch_count(h):
    return lib().sas_launch_count(h)


def sas_set_wait_limit(h, cycles):
    """Failure-path diagnostics: main-loop wait budget in SM cycles (0: default)."""
    _check(lib().sas_set_wait_limit(h, int(cycles)), h, "sas_set_wait_limit")


def sas_get_tile_union_counts(h, n):
    out = (ctypes.c_int32 * n)()
    _check(lib().sas_get_tile_union_counts(h, out, n), h, "sas_get_tile_union_counts")
    return list(out)


def sas_get_attention_work(h):
    """(tiles, tile_blocks) of the last attention forward (see sas.h)."""
    t, b = ctypes.c_int64(0), ctypes.c_int64(0)
    _check(lib().sas_get_attention_work(h, ctypes.byref(t), ctypes.byref(b)), h, "sas_get_attention_work")
    return t.value, b.value


def sas_selftest_wait_timeout(limit_cycles):
    v = ctypes.c_int32(-1)
    _check(lib().sas_selftest_wait_timeout(int(limit_cycles), ctypes.byref(v)), None, "sas_selftest_wait_timeout")
    return v.value


class SasLayer:
    """Owns one handle; allocates outputs and calls the C ABI."""

    def __init__(self, B, H, N, d, topk, mode=SAS_MODE_TRAIN_SOFT, selector=SAS_SEL_SCORES_GIVEN, d_sel=0,
                 sm_scale=0.0, gate_act=SAS_GATE_SOFTMAX, gate_pos=SAS_GATE_INNER, Hkv=0, max_seqs=0, max_seqlen=0,
                 scope=SAS_SCOPE_SPARSE):
        self.B, self.H, self.N, self.d, self.topk = B, H, N, d, topk
        self.mode = mode
        self.Hkv = Hkv or H                      # kept lists are per KV group
        self.selector = selector
        self.scope = scope
        self.h = sas_create(B, H, N, d, topk, mode, selector, d_sel, sm_scale, 64, gate_act, gate_pos, Hkv,
                            max_seqs, max_seqlen, scope)

    def attention_varlen(self, cu_seqlens, Q, K, V, scores=None, want_sel=True, stream=None, sel_fill=-1, Wq=None,
                         Wk=None):
        """Packed sequences (handle made with max_seqs > 0): Q [H, N, d], K/V [Hkv, N, d],
        scores [Hkv, N, C] (or the learned selector's Wq, Wk), cu_seqlens int32 on the
        device.  The library does not write rows past cu[-1]: they keep the fill of
        the tensors made here (0, and sel_fill in sel_idx)."""
        dev = Q.device
        O = torch.zeros_like(Q)
        LSE = torch.zeros(self.H, self.N, device=dev, dtype=torch.float32)
        sel_idx = sel_logg = None
        if want_sel:
            k = max(self.topk, 1)
            sel_idx = torch.full((self.Hkv, self.N, k), sel_fill, device=dev, dtype=torch.int32)
            sel_logg = torch.zeros(self.Hkv, self.N, k, device=dev, dtype=torch.float32)
        sas_attention_fwd_varlen(self.h, cu_seqlens, Q, K, V, scores, O, LSE, sel_idx, sel_logg, stream, Wq, Wk)
        return O, LSE, sel_idx, sel_logg

    def _outputs(self, Q, want_sel):
        dev = Q.device
        O = torch.empty_like(Q)
        LSE = torch.empty(self.B, self.H, self.N, device=dev, dtype=torch.float32)
        sel_idx = sel_logg = None
        if want_sel and self.scope == SAS_SCOPE_SPARSE:
            k = max(self.topk, 1)
            sel_idx = torch.empty(self.B, self.Hkv, self.N, k, device=dev, dtype=torch.int32)
            sel_logg = torch.empty(self.B, self.Hkv, self.N, k, device=dev, dtype=torch.float32)
        return O, LSE, sel_idx, sel_logg

    def attention(self, Q, K, V, scores=None, Wq=None, Wk=None, want_sel=True, stream=None):
        """Returns (O, LSE, sel_idx, sel_logg); the full scope keeps no Top-K (sel_* None)."""
        O, LSE, sel_idx, sel_logg = self._outputs(Q, want_sel)
        sas_attention_fwd(self.h, Q, K, V, O, scores, Wq, Wk, LSE, sel_idx, sel_logg, stream)
        return O, LSE, sel_idx, sel_logg

    def attention_noisy(self, Q, K, V, noise, scores=None, Wq=None, Wk=None, want_sel=True, stream=None):
        """full*: the scores plus `noise` (fp32, the layout of given scores) choose and gate the blocks."""
        O, LSE, sel_idx, sel_logg = self._outputs(Q, want_sel)
        sas_attention_fwd_noisy(self.h, Q, K, V, O, noise, scores, Wq, Wk, LSE, sel_idx, sel_logg, stream)
        return O, LSE, sel_idx, sel_logg

    def attention_bwd(self, Q, K, V, O, LSE, dO, scores=None, sel_idx=None, sel_logg=None, want_ds=False,
                      stream=None):
        """Returns (dQ, dK, dV, dlogg, dscores); dscores only with want_ds (given scores).
        With Hkv < H, dK, dV, dlogg and dscores are per KV group (sums over its heads).
        The full scope and the hard-STE mode report dlogg for every block: [B, Hkv, N, C]."""
        dQ, dK, dV = torch.empty_like(Q), torch.empty_like(K), torch.empty_like(V)
        C = -(-self.N // 64)
        width = C if (self.scope == SAS_SCOPE_FULL or self.mode == SAS_MODE_TRAIN_HARD_STE) else max(self.topk, 1)
        dlogg = torch.empty(self.B, self.Hkv, self.N, width, device=Q.device, dtype=torch.float32)
        ds = None
        if want_ds:
            ds = torch.empty(self.B, self.Hkv, self.N, -(-self.N // 64), device=Q.device, dtype=torch.float32)
        sas_attention_bwd(self.h, Q, K, V, O, LSE, dO, dQ, dK, dV, scores, sel_idx, sel_logg, dlogg, ds, stream)
        return dQ, dK, dV, dlogg, ds

    def attention_bwd_varlen(self, Q, K, V, O, LSE, dO, scores=None, sel_idx=None, sel_logg=None, want_ds=False,
                             stream=None):
        """Backward of the last attention_varlen on this handle: Q, O, dO [H, N, d],
        K, V [Hkv, N, d].  Returns (dQ, dK, dV, dlogg [Hkv, N, topk], dscores [Hkv, N, C]
        or None); rows past cu[-1] keep the zero fill of the tensors made here."""
        dev = Q.device
        dQ, dK, dV = torch.zeros_like(Q), torch.zeros_like(K), torch.zeros_like(V)
        dlogg = torch.zeros(self.Hkv, self.N, max(self.topk, 1), device=dev, dtype=torch.float32)
        ds = None
        if want_ds:
            ds = torch.zeros(self.Hkv, self.N, scores.shape[-1], device=dev, dtype=torch.float32)
        sas_attention_bwd(self.h, Q, K, V, O, LSE, dO, dQ, dK, dV, scores, sel_idx, sel_logg, dlogg, ds, stream)
        return dQ, dK, dV, dlogg, ds

    def qk_norm_rope(self, qkv, wq, wk, cos, sin, positions=None, eps=1e-6, interleaved=False, out=None, stream=None):
        """Per-head norm of queries and keys and the rotary rotation: the fused projection qkv
        [B, N, H + 2 Hkv, d] to (Q [B, H, N, d], K, V [B, Hkv, N, d]), as attention() takes them; out reuses the
        caller's."""
        if out is None:
            with _on(stream):
                Q = torch.empty(self.B, self.H, self.N, self.d, device=qkv.device, dtype=torch.bfloat16)
                K = torch.empty(self.B, self.Hkv, self.N, self.d, device=qkv.device, dtype=torch.bfloat16)
                out = (Q, K, torch.empty_like(K))
        sas_qk_norm_rope_fwd(self.h, qkv, wq, wk, cos, sin, *out, positions, eps, interleaved, stream)
        return out

    def qk_norm_rope_bwd(self, qkv, wq, wk, cos, sin, dQ, dK, dV, positions=None, eps=1e-6, interleaved=False, out=None,
                         stream=None):
        """Returns (dqkv [B, N, H + 2 Hkv, d] bf16, dwq, dwk fp32 [d]); out reuses the caller's."""
        if out is None:
            with _on(stream):
                dqkv = torch.empty(qkv.shape, device=qkv.device, dtype=torch.bfloat16)
                dwq = torch.empty(self.d, device=qkv.device, dtype=torch.float32)
                out = (dqkv, dwq, torch.empty_like(dwq))
        sas_qk_norm_rope_bwd(self.h, qkv, wq, wk, cos, sin, dQ, dK, dV, *out, positions, eps, interleaved, stream)
        return out

    def mlp(self, X, W1, W2, b1=None, b2=None, stream=None):
        Y = torch.empty(X.shape[0], W2.shape[0], device=X.device, dtype=torch.bfloat16)
        sas_mlp_fwd(self.h, X, W1, W2, Y, b1, b2, stream)
        return Y

    def close(self):
        if self.h is not None:
            sas_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ------------------------------------------------------------------ decode


def _dcheck(status, handle, what):
    if status != SAS_OK:
        L = lib()
        msg = L.sas_status_str(status).decode()
        if handle is not None:
            detail = L.sas_decode_last_error(handle).decode()
            if detail:
                msg += ": " + detail
        raise SasError(status, f"{what}: {msg}")


def sas_decode_create(B, Hq, Hkv, d, topk, max_blocks, num_pages, d_sel=0, sm_scale=0.0, dense=False, block=64):
    cfg = SasDecodeConfig(B, Hq, Hkv, d, d_sel, block, topk, max_blocks, num_pages, sm_scale, 1 if dense else 0)
    h = ctypes.c_void_p()
    _dcheck(lib().sas_decode_create(ctypes.byref(cfg), ctypes.byref(h)), None, "sas_decode_create")
    return h


def sas_decode_create_status(B, Hq, Hkv, d, topk, max_blocks, num_pages, d_sel=0, sm_scale=0.0, dense=0, block=64):
    """Raw status of sas_decode_create (argument-check tests); destroys the handle on success."""
    cfg = SasDecodeConfig(B, Hq, Hkv, d, d_sel, block, topk, max_blocks, num_pages, sm_scale, dense)
    h = ctypes.c_void_p()
    st = lib().sas_decode_create(ctypes.byref(cfg), ctypes.byref(h))
    if st == SAS_OK:
        lib().sas_decode_destroy(h)
    return st


def sas_decode_destroy(h):
    lib().sas_decode_destroy(h)


def sas_decode_summarize(h, K_cache, block_table, seq_lens, Wk, Ksum, stream=None):
    bf, i32 = torch.bfloat16, torch.int32
    st = lib().sas_decode_summarize(h, _ptr(K_cache, bf, "K_cache"), _ptr(block_table, i32, "block_table"),
                                    _ptr(seq_lens, i32, "seq_lens"), _ptr(Wk, bf, "Wk"), _ptr(Ksum, bf, "Ksum"),
                                    _stream(stream))
    _dcheck(st, h, "sas_decode_summarize")


def sas_decode_step(h, q, K_cache, V_cache, block_table, seq_lens, O, k_new=None, v_new=None, Wq=None, Wk=None,
                    Ksum=None, LSE=None, sel_idx=None, stream=None):
    bf, i32 = torch.bfloat16, torch.int32
    st = lib().sas_decode_step(
        h, _ptr(q, bf, "q"), _ptr(k_new, bf, "k_new", False), _ptr(v_new, bf, "v_new", False),
        _ptr(K_cache, bf, "K_cache"), _ptr(V_cache, bf, "V_cache"), _ptr(block_table, i32, "block_table"),
        _ptr(seq_lens, i32, "seq_lens"), _ptr(Wq, bf, "Wq", False), _ptr(Wk, bf, "Wk", False),
        _ptr(Ksum, bf, "Ksum", False), _ptr(O, bf, "O"), _ptr(LSE, torch.float32, "LSE", False),
        _ptr(sel_idx, i32, "sel_idx", False), _stream(stream))
    _dcheck(st, h, "sas_decode_step")


def sas_decode_get_device_status(h):
    v = ctypes.c_int32(0)
    _dcheck(lib().sas_decode_get_device_status(h, ctypes.byref(v)), h, "sas_decode_get_device_status")
    return v.value


def sas_decode_set_timing(h, enable):
    _dcheck(lib().sas_decode_set_timing(h, 1 if enable else 0), h, "sas_decode_set_timing")


def sas_decode_get_timings(h):
    n = SAS_DECODE_NUM_KERNEL_KINDS
    launches = (ctypes.c_int64 * n)()
    ms = (ctypes.c_double * n)()
    _dcheck(lib().sas_decode_get_timings(h, launches, ms, n), h, "sas_decode_get_timings")
    return {DECODE_KERNEL_KINDS[k]: (launches[k], ms[k]) for k in range(n)}


def sas_decode_launch_count(h):
    return lib().sas_decode_launch_count(h)


class SasDecoder:
    """Owns one decode handle; allocates the step's outputs and calls the C ABI."""

    def __init__(self, B, Hq, Hkv, d, topk, max_blocks, num_pages, d_sel=0, sm_scale=0.0, dense=False):
        self.B, self.Hq, self.Hkv, self.d, self.topk = B, Hq, Hkv, d, topk
        self.dense = dense
        self.h = sas_decode_create(B, Hq, Hkv, d, topk, max_blocks, num_pages, d_sel, sm_scale, dense)

    def summarize(self, K_cache, block_table, seq_lens, Wk, Ksum, stream=None):
        sas_decode_summarize(self.h, K_cache, block_table, seq_lens, Wk, Ksum, stream)

    def step(self, q, K_cache, V_cache, block_table, seq_lens, k_new=None, v_new=None, Wq=None, Wk=None, Ksum=None,
             out=None, stream=None):
        """Returns (O, LSE, sel_idx); sel_idx is None in dense mode.  out = (O, LSE, sel_idx)
        reuses caller buffers (as a captured graph needs)."""
        if out is None:
            O = torch.empty(self.B, self.Hq, self.d, device=q.device, dtype=torch.bfloat16)
            LSE = torch.empty(self.B, self.Hq, device=q.device, dtype=torch.float32)
            sel = None if self.dense else torch.empty(self.B, self.Hkv, max(self.topk, 1), device=q.device,
                                                      dtype=torch.int32)
        else:
            O, LSE, sel = out
        sas_decode_step(self.h, q, K_cache, V_cache, block_table, seq_lens, O, k_new, v_new, Wq, Wk, Ksum, LSE,
                        sel, stream)
        return O, LSE, sel

    def close(self):
        if self.h is not None:
            sas_decode_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ------------------------------------------------------------------ serving step


def _ccheck(status, handle, what):
    if status != SAS_OK:
        L = lib()
        msg = L.sas_status_str(status).decode()
        if handle is not None:
            detail = L.sas_chunk_last_error(handle).decode()
            if detail:
                msg += ": " + detail
        raise SasError(status, f"{what}: {msg}")


def sas_chunk_create(max_seqs, Hq, Hkv, d, max_blocks, num_pages, max_tokens, sm_scale=0.0, block=64):
    cfg = SasChunkConfig(max_seqs, Hq, Hkv, d, block, max_blocks, num_pages, max_tokens, sm_scale)
    h = _Handle()
    _ccheck(lib().sas_chunk_create(ctypes.byref(cfg), ctypes.byref(h)), None, "sas_chunk_create")
    h.sizes = Hq, d, max_blocks, (num_pages, Hkv, block, d)
    return h


def sas_chunk_create_status(max_seqs, Hq, Hkv, d, max_blocks, num_pages, max_tokens, sm_scale=0.0, block=64):
    """Raw status of sas_chunk_create (argument-check tests); destroys the handle on success."""
    cfg = SasChunkConfig(max_seqs, Hq, Hkv, d, block, max_blocks, num_pages, max_tokens, sm_scale)
    h = ctypes.c_void_p()
    st = lib().sas_chunk_create(ctypes.byref(cfg), ctypes.byref(h))
    if st == SAS_OK:
        lib().sas_chunk_destroy(h)
    return st


def sas_chunk_destroy(h):
    lib().sas_chunk_destroy(h)


def _table(h, block_table, B):
    if block_table.shape != (B, _sizes(h)[2]):
        raise ValueError(f"block_table must have {B} rows and {_sizes(h)[2]} columns, got {tuple(block_table.shape)}")


def sas_chunk_plan(h, seq_lens, new_lens, free_pages, free_begin, block_table, kv_lens, cu_new, positions, slots,
                   free_end, held_lens=None, stream=None):
    i32, B, T, dev = torch.int32, seq_lens.shape[0], positions.shape[0], seq_lens.get_device()
    _table(h, block_table, B)
    st = lib().sas_chunk_plan(
        h, B, T, _arg(seq_lens, i32, "seq_lens", dev, (B,)), _arg(new_lens, i32, "new_lens", dev, (B,)),
        None if held_lens is None else _arg(held_lens, i32, "held_lens", dev, (B,)),
        _arg(free_pages, i32, "free_pages", dev), free_pages.numel(), _arg(free_begin, i32, "free_begin", dev, (1,)),
        _arg(block_table, i32, "block_table", dev), _arg(kv_lens, i32, "kv_lens", dev, (B,)),
        _arg(cu_new, i32, "cu_new", dev, (B + 1,)), _arg(positions, i32, "positions", dev, (T,)),
        _arg(slots, torch.int64, "slots", dev, (T,)), _arg(free_end, i32, "free_end", dev, (1,)), _raw_stream(stream, dev))
    if st != SAS_OK:
        _ccheck(st, h, "sas_chunk_plan")


def sas_chunk_append(h, qkv, wq, wk, cos, sin, positions, slots, Q, K_cache, V_cache, eps=1e-6, interleaved=False,
                     stream=None):
    """qkv [T, Hq + 2 Hkv, d] (tokens evenly spaced, any distance)."""
    Hq, d, _, cache = _sizes(h)
    T, Hkv, dev, bf, f32 = Q.shape[0], cache[1], Q.get_device(), torch.bfloat16, torch.float32
    cfg = _rope_config(cos, eps, interleaved)
    st = lib().sas_chunk_append(
        h, cfg, T, _rows(qkv, bf, "qkv", dev, (T, Hq + 2 * Hkv, d)), _token_stride(qkv, "qkv", 1),
        _arg(wq, bf, "wq", dev, (d,)), _arg(wk, bf, "wk", dev, (d,)), _arg(cos, f32, "cos", dev), _arg(sin, f32, "sin", dev, cos.shape),
        _arg(positions, torch.int32, "positions", dev, (T,)), _arg(slots, torch.int64, "slots", dev, (T,)),
        _arg(Q, bf, "Q", dev, (T, Hq, d)), _arg(K_cache, bf, "K_cache", dev, cache), _arg(V_cache, bf, "V_cache", dev, cache),
        _raw_stream(stream, dev))
    if st != SAS_OK:
        _ccheck(st, h, "sas_chunk_append")


def sas_chunk_attention(h, Q, K_cache, V_cache, block_table, cu_new, kv_lens, O, LSE=None, stream=None):
    i32, bf, B, T, dev = torch.int32, torch.bfloat16, kv_lens.shape[0], Q.shape[0], Q.get_device()
    _table(h, block_table, B)
    Hq, d, _, cache = _sizes(h)
    st = lib().sas_chunk_attention(
        h, B, T, _arg(Q, bf, "Q", dev, (T, Hq, d)), _arg(K_cache, bf, "K_cache", dev, cache),
        _arg(V_cache, bf, "V_cache", dev, cache), _arg(block_table, i32, "block_table", dev),
        _arg(cu_new, i32, "cu_new", dev, (B + 1,)), _arg(kv_lens, i32, "kv_lens", dev, (B,)), _arg(O, bf, "O", dev, Q.shape),
        None if LSE is None else _arg(LSE, torch.float32, "LSE", dev, Q.shape[:2]), _raw_stream(stream, dev))
    if st != SAS_OK:
        _ccheck(st, h, "sas_chunk_attention")


def _prob_rows(t, name, rows, dev, V):
    """Address and row stride of an fp32 [rows, V] tensor with contiguous columns."""
    at = _rows(t, torch.float32, name, dev, (rows, V))
    st = t.stride()
    if V > 1 and st[1] != 1:
        raise ValueError(f"{name} must have contiguous columns")
    return at, st[0] if rows > 1 else max(st[0], V)


def sas_chunk_verify(h, tokens, cu_draft, target, draft, u, noise, accepted, out_tokens, stream=None):
    """draft None: the drafts were certain."""
    i32, B, n, V, dev = torch.int32, cu_draft.shape[0] - 1, tokens.shape[0], target.shape[1], target.get_device()
    p, ldp = _prob_rows(target, "target", n + B, dev, V)
    q, ldq = (None, V) if draft is None else _prob_rows(draft, "draft", n, dev, V)
    e, lde = _prob_rows(noise, "noise", B, dev, V)
    if out_tokens.dim() != 2 or out_tokens.shape[0] != B or out_tokens.shape[1] < 1:
        raise ValueError(f"out_tokens must have {B} rows and at least one column")
    st = lib().sas_chunk_verify(
        h, B, n, out_tokens.shape[1] - 1, V, _arg(tokens, i32, "tokens", dev, (n,)), _arg(cu_draft, i32, "cu_draft", dev, (B + 1,)), p,
        ldp, q, ldq, _arg(u, torch.float32, "u", dev, (n,)), e, lde, _arg(accepted, i32, "accepted", dev, (B,)),
        _arg(out_tokens, i32, "out_tokens", dev), _raw_stream(stream, dev))
    if st != SAS_OK:
        _ccheck(st, h, "sas_chunk_verify")


def sas_chunk_get_device_status(h):
    v = ctypes.c_int32(0)
    _ccheck(lib().sas_chunk_get_device_status(h, ctypes.byref(v)), h, "sas_chunk_get_device_status")
    return v.value


def sas_chunk_set_timing(h, enable):
    _ccheck(lib().sas_chunk_set_timing(h, 1 if enable else 0), h, "sas_chunk_set_timing")


def sas_chunk_get_timings(h):
    n = SAS_CHUNK_NUM_KERNEL_KINDS
    launches = (ctypes.c_int64 * n)()
    ms = (ctypes.c_double * n)()
    _ccheck(lib().sas_chunk_get_timings(h, launches, ms, n), h, "sas_chunk_get_timings")
    return {CHUNK_KERNEL_KINDS[k]: (launches[k], ms[k]) for k in range(n)}


def sas_chunk_launch_count(h):
    return lib().sas_chunk_launch_count(h)


def sas_chunk_set_wait_limit(h, cycles):
    """Failure-path diagnostics: wait budget of the attention in SM cycles (0: default)."""
    _ccheck(lib().sas_chunk_set_wait_limit(h, int(cycles)), h, "sas_chunk_set_wait_limit")


# Outputs of a page plan (see sas_chunk_plan in sas.h).
ChunkPlan = collections.namedtuple("ChunkPlan", "kv_lens cu_new positions slots free_end")


class SasChunk:
    """One serving step over a paged cache: plan -> append -> attention (-> verify).

    Owns one handle; allocates the outputs (on the stream the call runs on) unless the caller
    passes its own, as a captured graph needs.  K_cache, V_cache [num_pages, Hkv, 64, d] and
    block_table [requests, max_blocks] are those of SasDecoder."""

    def __init__(self, max_seqs, Hq, Hkv, d, max_blocks, num_pages, max_tokens, sm_scale=0.0):
        self.Hq, self.Hkv, self.d, self.max_blocks = Hq, Hkv, d, max_blocks
        self.cache_shape = (num_pages, Hkv, 64, d)
        self.h = sas_chunk_create(max_seqs, Hq, Hkv, d, max_blocks, num_pages, max_tokens, sm_scale)

    def plan_buffers(self, num_seqs, T, device):
        i32 = torch.int32
        return ChunkPlan(torch.empty(num_seqs, device=device, dtype=i32), torch.empty(num_seqs + 1, device=device, dtype=i32),
                         torch.empty(T, device=device, dtype=i32), torch.empty(T, device=device, dtype=torch.int64),
                         torch.empty(1, device=device, dtype=i32))

    def plan(self, seq_lens, new_lens, free_pages, free_begin, block_table, T, held_lens=None, out=None, stream=None):
        """Pages and slots of the new tokens: a ChunkPlan; block_table gets the new pages.  T: capacity for new
        tokens (positions and slots are -1 past their number).  held_lens: tokens whose pages each request holds
        (seq_lens if not given)."""
        if out is None:
            with _on(stream):
                out = self.plan_buffers(seq_lens.shape[0], T, seq_lens.device)
        elif out.positions.shape[0] != T:
            raise ValueError(f"out.positions must have {T} entries")
        sas_chunk_plan(self.h, seq_lens, new_lens, free_pages, free_begin, block_table, *out, held_lens, stream)
        return out

    def append(self, qkv, wq, wk, cos, sin, positions, slots, K_cache, V_cache, eps=1e-6, interleaved=False, out=None,
               stream=None):
        """Norm + rotation of the new tokens' queries and keys; keys and values into the cache.  Returns Q
        [T, Hq, d] (rows of slot -1 are not written)."""
        if out is None:
            with _on(stream):
                out = torch.empty(qkv.shape[0], self.Hq, self.d, device=qkv.device, dtype=torch.bfloat16)
        sas_chunk_append(self.h, qkv, wq, wk, cos, sin, positions, slots, out, K_cache, V_cache, eps, interleaved, stream)
        return out

    def attention(self, Q, K_cache, V_cache, block_table, cu_new, kv_lens, out=None, stream=None):
        """Dense causal attention of the new tokens.  Returns (O [T, Hq, d], LSE [T, Hq]); out = (O, LSE) reuses
        caller buffers (LSE may be None)."""
        if out is None:
            with _on(stream):
                out = (torch.empty_like(Q), torch.empty(Q.shape[:2], device=Q.device, dtype=torch.float32))
        sas_chunk_attention(self.h, Q, K_cache, V_cache, block_table, cu_new, kv_lens, out[0], out[1], stream)
        return out

    def verify(self, tokens, cu_draft, target, draft, u, noise, max_draft, out=None, stream=None):
        """Accepted drafts and the next token of every request: (accepted [requests], tokens [requests, max_draft + 1]
        padded with -1)."""
        B = cu_draft.shape[0] - 1
        if out is None:
            with _on(stream):
                out = (torch.empty(B, device=target.device, dtype=torch.int32),
                       torch.empty(B, max_draft + 1, device=target.device, dtype=torch.int32))
        elif out[1].dim() != 2 or out[1].shape[1] != max_draft + 1:
            raise ValueError(f"out[1] must have {max_draft + 1} columns")
        sas_chunk_verify(self.h, tokens, cu_draft, target, draft, u, noise, out[0], out[1], stream)
        return out

    def close(self):
        if self.h is not None:
            sas_chunk_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
