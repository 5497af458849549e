"""ctypes binding of libvista.so: argument marshalling only.

The functions carry the names of the C entry points declared in
include/vista.h and do nothing but turn torch tensors (device memory) and the
current torch stream into the pointers the C ABI takes.  Every step of the
computation runs inside the library's HIP kernels; when the library is absent
or fails to load, importing this module's entry points raises -- there is no
CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libvista.so")

VISTA_OK = 0
VISTA_ERR_NULL, VISTA_ERR_SHAPE, VISTA_ERR_OFFSETS = 1, 2, 3
VISTA_ERR_UNSUPPORTED, VISTA_ERR_WORKSPACE, VISTA_ERR_HIP, VISTA_ERR_SCRATCH = 4, 5, 6, 7
VISTA_STATIC_SCRATCH_BYTES = 64 << 20
VISTA_F32, VISTA_BF16 = 0, 1
VISTA_ATTN_SOFTMAX, VISTA_ATTN_SILU, VISTA_ATTN_QLA = 0, 1, 2
VISTA_FLAG_SELF_TERM = 1

EXPORTS = (
    "vista_status_string",
    "vista_summarize_segment_items",
    "vista_summarize_call_segment_items",
    "vista_summarize_workspace_bytes",
    "vista_summarize_schedule",
    "vista_summarize",
    "vista_summarize_static",
    "vista_target_attend",
    "vista_target_attend_q8",
    "vista_quantize_summaries",
    "vista_summarize_q8",
    "vista_qla_backward_workspace_bytes",
    "vista_qla_backward",
    "vista_summarize_backward_workspace_bytes",
    "vista_summarize_backward",
    "vista_target_attend_backward_workspace_bytes",
    "vista_target_attend_backward",
    "vista_layer_norm",
    "vista_layer_norm_backward_workspace_bytes",
    "vista_layer_norm_backward",
    "vista_sglu_ffn",
)


class SummarizeDesc(C.Structure):
    _fields_ = [("B", C.c_int32), ("S", C.c_int32), ("d", C.c_int32), ("H", C.c_int32),
                ("dtype", C.c_int32), ("attn", C.c_int32), ("scale", C.c_float),
                ("segment_items", C.c_int32), ("total_items", C.c_int64),
                ("q_user_stride", C.c_int64), ("flags", C.c_int32), ("reserved", C.c_int32)]


class AttendDesc(C.Structure):
    _fields_ = [("B", C.c_int32), ("C", C.c_int32), ("S", C.c_int32), ("d", C.c_int32),
                ("H", C.c_int32), ("dtype", C.c_int32), ("scale", C.c_float), ("flags", C.c_int32)]


class CodecDesc(C.Structure):
    _fields_ = [("rows", C.c_int64), ("d", C.c_int32), ("H", C.c_int32), ("dtype", C.c_int32)]


class FfnDesc(C.Structure):
    _fields_ = [("rows", C.c_int64), ("d", C.c_int32), ("d_ff", C.c_int32),
                ("dtype", C.c_int32), ("eps", C.c_float)]


class NormDesc(C.Structure):
    _fields_ = [("rows", C.c_int64), ("d", C.c_int32), ("dtype", C.c_int32), ("eps", C.c_float)]


class VistaError(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        super().__init__(lib().vista_status_string(status).decode())


_lib = None


def lib() -> C.CDLL:
    """Loads libvista.so (built by ``python -m paper_2510_22049_amd.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} is missing: run `python -m paper_2510_22049_amd.build` first; "
            "there is no fallback path")
    L = C.CDLL(LIB_PATH)
    vp, i64p = C.c_void_p, C.POINTER(C.c_int64)
    L.vista_status_string.restype = C.c_char_p
    L.vista_status_string.argtypes = [C.c_int]
    L.vista_summarize_segment_items.restype = C.c_int32
    L.vista_summarize_segment_items.argtypes = [C.POINTER(SummarizeDesc)]
    L.vista_summarize_call_segment_items.restype = C.c_int32
    L.vista_summarize_call_segment_items.argtypes = [C.POINTER(SummarizeDesc), C.c_size_t]
    L.vista_summarize_workspace_bytes.restype = C.c_size_t
    L.vista_summarize_workspace_bytes.argtypes = [C.POINTER(SummarizeDesc)]
    L.vista_summarize_schedule.restype = C.c_int64
    L.vista_summarize_schedule.argtypes = [C.POINTER(SummarizeDesc), i64p, i64p, C.c_int64]
    L.vista_summarize.restype = C.c_int
    L.vista_summarize.argtypes = [C.POINTER(SummarizeDesc), vp, vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
    L.vista_summarize_static.restype = C.c_int
    L.vista_summarize_static.argtypes = [C.POINTER(SummarizeDesc), vp, vp, vp, vp, vp, vp, vp, vp]
    L.vista_summarize_q8.restype = C.c_int
    L.vista_summarize_q8.argtypes = [C.POINTER(SummarizeDesc), vp, vp, vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
    L.vista_qla_backward_workspace_bytes.restype = C.c_size_t
    L.vista_qla_backward_workspace_bytes.argtypes = [C.POINTER(SummarizeDesc)]
    L.vista_qla_backward.restype = C.c_int
    L.vista_qla_backward.argtypes = [C.POINTER(SummarizeDesc)] + [vp] * 13 + [C.c_size_t, vp]
    L.vista_summarize_backward_workspace_bytes.restype = C.c_size_t
    L.vista_summarize_backward_workspace_bytes.argtypes = [C.POINTER(SummarizeDesc)]
    L.vista_summarize_backward.restype = C.c_int
    L.vista_summarize_backward.argtypes = [C.POINTER(SummarizeDesc)] + [vp] * 13 + [C.c_size_t, vp]
    L.vista_target_attend_backward_workspace_bytes.restype = C.c_size_t
    L.vista_target_attend_backward_workspace_bytes.argtypes = [C.POINTER(AttendDesc)]
    L.vista_target_attend_backward.restype = C.c_int
    L.vista_target_attend_backward.argtypes = [C.POINTER(AttendDesc)] + [vp] * 6 + [C.c_size_t, vp]
    L.vista_layer_norm.restype = C.c_int
    L.vista_layer_norm.argtypes = [C.POINTER(NormDesc)] + [vp] * 5
    L.vista_layer_norm_backward_workspace_bytes.restype = C.c_size_t
    L.vista_layer_norm_backward_workspace_bytes.argtypes = [C.POINTER(NormDesc)]
    L.vista_layer_norm_backward.restype = C.c_int
    L.vista_layer_norm_backward.argtypes = [C.POINTER(NormDesc)] + [vp] * 7 + [C.c_size_t, vp]
    L.vista_quantize_summaries.restype = C.c_int
    L.vista_quantize_summaries.argtypes = [C.POINTER(CodecDesc), vp, vp, vp, vp]
    L.vista_target_attend_q8.restype = C.c_int
    L.vista_target_attend_q8.argtypes = [C.POINTER(AttendDesc), vp, vp, vp, vp, vp]
    L.vista_target_attend.restype = C.c_int
    L.vista_target_attend.argtypes = [C.POINTER(AttendDesc), vp, vp, vp, vp]
    L.vista_sglu_ffn.restype = C.c_int
    L.vista_sglu_ffn.argtypes = [C.POINTER(FfnDesc), vp, vp, vp, vp, vp, vp]
    _lib = L
    return L


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return VISTA_F32
    if t.dtype == torch.bfloat16:
        return VISTA_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _dev(t: torch.Tensor, name: str) -> int:
    if not t.is_cuda:
        raise ValueError(f"{name} must live in device memory")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _shaped(like: torch.Tensor, tensors) -> None:
    """Each (name, tensor, shape) has that shape, the type of `like` and its device, which is the current one (the call goes to
    the current device's stream), and is contiguous: a kernel would otherwise read or write past the end of one of them.
    A tensor that is None is left out."""
    dtype, index = like.dtype, like.get_device()
    if index >= 0 and index == _device():
        for _, t, shape in tensors:              # the usual case: every check at once, half of a small call's host time otherwise
            if t is not None and (t.dtype is not dtype or t.get_device() != index or t.shape != shape or not t.is_contiguous()):
                break
        else:
            return
    elif index >= 0:
        raise ValueError("the tensors live on another device than the current one")
    for name, t, shape in tensors:
        if t is None:
            continue
        if tuple(t.shape) != tuple(shape):
            raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
        if t.dtype != dtype:
            raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
        if t.device != like.device:
            raise ValueError(f"{name} must live on {like.device}")
    for name, t, _ in tensors:
        if t is not None:
            _dev(t, name)


def _workspace(workspace, need, like: torch.Tensor) -> torch.Tensor:
    """The caller's workspace, or one of torch's of need() bytes where there is none."""
    if workspace is None:
        return torch.empty(max(need(), 256), dtype=torch.uint8, device=like.device)
    if workspace.dtype is not torch.uint8 or workspace.get_device() != like.get_device():
        raise ValueError(f"workspace must be uint8 on {like.device}")
    return workspace


def _at(t):
    """Address of a tensor that _shaped has checked, or None."""
    return None if t is None else t.data_ptr()


def _stream_getter():
    """A function that gives the current stream of the current device as a hipStream_t.  torch.cuda.current_stream() builds a
    Stream object for it (2.8 us, more than half of a small call's host time), the two private functions take 0.2; a torch
    that does not have them goes the public way."""
    raw, device = (getattr(torch._C, n, None) for n in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))
    if raw is None or device is None:
        return lambda: torch.cuda.current_stream().cuda_stream
    return lambda: raw(device())


_stream = _stream_getter()
_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def summarize_desc(B, S, d, H, dtype, total_items, per_user_q=False, scale=0.0, segment_items=0,
                   attn=VISTA_ATTN_SOFTMAX, self_term=False):
    return SummarizeDesc(B=B, S=S, d=d, H=H, dtype=dtype, attn=attn, scale=scale,
                         segment_items=segment_items, total_items=total_items,
                         q_user_stride=S * d if per_user_q else 0,
                         flags=VISTA_FLAG_SELF_TERM if self_term else 0, reserved=0)


def vista_summarize_segment_items(desc: SummarizeDesc) -> int:
    return lib().vista_summarize_segment_items(C.byref(desc))


def vista_summarize_call_segment_items(desc: SummarizeDesc, workspace_bytes: int = 0) -> int:
    return lib().vista_summarize_call_segment_items(C.byref(desc), workspace_bytes)


def vista_summarize_workspace_bytes(desc: SummarizeDesc) -> int:
    return lib().vista_summarize_workspace_bytes(C.byref(desc))


def vista_summarize_schedule(desc: SummarizeDesc, offsets_host):
    """The tiles the kernels visit, int64 [n, 4] = (segment, user, first row, rows); host only.
    ``offsets_host`` is a numpy int64 array of B + 1 entries (not validated by the call)."""
    import numpy as np
    off = np.ascontiguousarray(offsets_host, dtype=np.int64)
    if off.size != desc.B + 1:
        raise ValueError("offsets_host must hold B + 1 entries")
    ptr = off.ctypes.data_as(C.POINTER(C.c_int64))
    n = lib().vista_summarize_schedule(C.byref(desc), ptr, None, 0)
    if n < 0:
        raise VistaError(VISTA_ERR_SHAPE)
    tiles = np.empty((n, 4), dtype=np.int64)
    lib().vista_summarize_schedule(C.byref(desc), ptr, tiles.ctypes.data_as(C.POINTER(C.c_int64)), n)
    return tiles


def vista_summarize(history_emb, offsets, virtual_queries, W_k, W_v, out, *, H, scale=0.0,
                    segment_items=0, offsets_host=None, workspace=None, attn=VISTA_ATTN_SOFTMAX,
                    self_term=False):
    """Stage 1.  history_emb [N,d], offsets int64 [B+1] (device), virtual_queries
    [S,d] or [B,S,d], W_k/W_v [d,d], out [B,S,d]; all on the GPU, same dtype.
    ``workspace`` is a uint8 device tensor (allocated here when None, by torch)."""
    B = offsets.numel() - 1
    S, d = virtual_queries.shape[-2:]
    N = history_emb.shape[0]
    desc = summarize_desc(B, S, d, H, _dtype_code(history_emb), N, virtual_queries.dim() == 3, scale,
                          segment_items, attn, self_term)
    if workspace is None:
        workspace = torch.empty(max(vista_summarize_workspace_bytes(desc), 256), dtype=torch.uint8, device=history_emb.device)
    host = None
    if offsets_host is not None:
        if offsets_host.is_cuda or offsets_host.dtype != torch.int64:
            raise ValueError("offsets_host must be a CPU int64 tensor")
        host = offsets_host.contiguous().data_ptr()
    if offsets.dtype != torch.int64:
        raise TypeError("offsets must be int64")
    st = lib().vista_summarize(C.byref(desc), _dev(history_emb, "history_emb") if N else None,
                               _dev(offsets, "offsets"), host, _dev(virtual_queries, "virtual_queries"),
                               _dev(W_k, "W_k"), _dev(W_v, "W_v"), _dev(out, "out"),
                               _dev(workspace, "workspace"), workspace.numel(), _stream())
    if st != VISTA_OK:
        raise VistaError(st)
    return workspace


def vista_summarize_q8(history_emb, offsets, virtual_queries, W_k, W_v, out_codes, out_scales, *, H, scale=0.0,
                       segment_items=0, offsets_host=None, workspace=None, attn=VISTA_ATTN_SOFTMAX, self_term=False):
    """Stage 1 with the cache codec fused: out_codes int8 [B,S,d], out_scales float32 [B,S,H]."""
    B = offsets.numel() - 1
    S, d = virtual_queries.shape[-2:]
    N = history_emb.shape[0]
    desc = summarize_desc(B, S, d, H, _dtype_code(history_emb), N, virtual_queries.dim() == 3, scale,
                          segment_items, attn, self_term)
    if workspace is None:
        workspace = torch.empty(max(vista_summarize_workspace_bytes(desc), 256), dtype=torch.uint8, device=history_emb.device)
    if out_codes.dtype != torch.int8 or out_scales.dtype != torch.float32:
        raise TypeError("out_codes must be int8 and out_scales float32")
    host = offsets_host.contiguous().data_ptr() if offsets_host is not None else None
    st = lib().vista_summarize_q8(C.byref(desc), _dev(history_emb, "history_emb") if N else None,
                                  _dev(offsets, "offsets"), host, _dev(virtual_queries, "virtual_queries"),
                                  _dev(W_k, "W_k"), _dev(W_v, "W_v"), _dev(out_codes, "out_codes"),
                                  _dev(out_scales, "out_scales"), _dev(workspace, "workspace"), workspace.numel(),
                                  _stream())
    if st != VISTA_OK:
        raise VistaError(st)
    return workspace


def vista_qla_backward(history_emb, offsets, virtual_queries, W_k, W_v, d_out, d_queries, d_keys, d_values, *, H,
                       segment_items=0, offsets_host=None, workspace=None, d_self_keys=None, d_self_values=None):
    """Gradients of quasi-linear attention: d_out [B,S,d] -> d_queries [B,S,d], d_keys / d_values [N,d];
    with d_self_keys / d_self_values [B,S,d] given, the forward had the self term and its gradients
    are formed as well."""
    B = offsets.numel() - 1
    S, d = virtual_queries.shape[-2:]
    N = history_emb.shape[0]
    self_term = d_self_keys is not None or d_self_values is not None
    desc = summarize_desc(B, S, d, H, _dtype_code(history_emb), N, virtual_queries.dim() == 3, 0.0,
                          segment_items, VISTA_ATTN_QLA, self_term)
    if workspace is None:
        workspace = torch.empty(max(lib().vista_qla_backward_workspace_bytes(C.byref(desc)), 256), dtype=torch.uint8, device=history_emb.device)
    host = offsets_host.contiguous().data_ptr() if offsets_host is not None else None
    st = lib().vista_qla_backward(C.byref(desc), _dev(history_emb, "history_emb") if N else None,
                                  _dev(offsets, "offsets"), host, _dev(virtual_queries, "virtual_queries"),
                                  _dev(W_k, "W_k"), _dev(W_v, "W_v"), _dev(d_out, "d_out"),
                                  _dev(d_queries, "d_queries"), _dev(d_keys, "d_keys") if N else None,
                                  _dev(d_values, "d_values") if N else None,
                                  _dev(d_self_keys, "d_self_keys") if d_self_keys is not None else None,
                                  _dev(d_self_values, "d_self_values") if d_self_values is not None else None,
                                  _dev(workspace, "workspace"), workspace.numel(), _stream())
    if st != VISTA_OK:
        raise VistaError(st)
    return workspace


def vista_summarize_backward(history_emb, offsets, virtual_queries, W_k, W_v, d_out, d_queries, d_keys, d_values, *, H,
                             scale=0.0, segment_items=0, offsets_host=None, workspace=None, d_self_keys=None,
                             d_self_values=None):
    """Gradients of softmax summarization: d_out [B,S,d] -> d_queries [B,S,d], d_keys / d_values [N,d] (of the projected
    keys and values); with d_self_keys and d_self_values [B,S,d] given, the forward had the self term and its gradients
    are formed as well.  Returns the workspace, which may be passed to the next call."""
    if offsets.dtype != torch.int64 or offsets.dim() != 1 or offsets.numel() < 2:
        raise TypeError("offsets must be int64 [B + 1]")
    if offsets.device != history_emb.device:
        raise ValueError("offsets must live where history_emb does")
    if virtual_queries.dim() not in (2, 3) or history_emb.dim() != 2:
        raise ValueError("history_emb must be [N, d] and virtual_queries [S, d] or [B, S, d]")
    B = offsets.numel() - 1
    S, d = virtual_queries.shape[-2:]
    N = history_emb.shape[0]
    per_user = virtual_queries.dim() == 3
    if (d_self_keys is None) != (d_self_values is None):
        raise ValueError("d_self_keys and d_self_values go together")
    items, user, summaries = (N, d), (B, S, d) if per_user else (S, d), (B, S, d)
    _shaped(history_emb, (("history_emb", history_emb, items), ("virtual_queries", virtual_queries, user), ("W_k", W_k, (d, d)),
                          ("W_v", W_v, (d, d)), ("d_out", d_out, summaries), ("d_queries", d_queries, summaries),
                          ("d_keys", d_keys, items), ("d_values", d_values, items), ("d_self_keys", d_self_keys, summaries),
                          ("d_self_values", d_self_values, summaries)))
    desc = summarize_desc(B, S, d, H, _dtype_code(history_emb), N, per_user, scale, segment_items, VISTA_ATTN_SOFTMAX,
                          d_self_keys is not None)
    host = None
    if offsets_host is not None:
        if offsets_host.is_cuda or offsets_host.dtype != torch.int64 or offsets_host.numel() != B + 1:
            raise ValueError("offsets_host must be a CPU int64 tensor of B + 1 entries")
        offsets_host = offsets_host.contiguous()
        host = offsets_host.data_ptr()
    workspace = _workspace(workspace, lambda: lib().vista_summarize_backward_workspace_bytes(C.byref(desc)), history_emb)
    st = lib().vista_summarize_backward(C.byref(desc), _at(history_emb if N else None), _dev(offsets, "offsets"), host,
                                        virtual_queries.data_ptr(), W_k.data_ptr(), W_v.data_ptr(), d_out.data_ptr(),
                                        d_queries.data_ptr(), _at(d_keys if N else None), _at(d_values if N else None),
                                        _at(d_self_keys), _at(d_self_values), _dev(workspace, "workspace"), workspace.numel(),
                                        _stream())
    if st != VISTA_OK:
        raise VistaError(st)
    return workspace


def vista_target_attend_backward(candidates, summaries, d_out, d_candidates, d_summaries, *, H, scale=0.0, self_term=False,
                                 workspace=None):
    """Gradients of candidate attention: d_out [B,C,d] -> d_candidates [B,C,d], d_summaries [B,S,d].  Returns the
    workspace, which may be passed to the next call."""
    if candidates.dim() != 3 or summaries.dim() != 3:
        raise ValueError("candidates must be [B, C, d] and summaries [B, S, d]")
    B, Cn, d = candidates.shape
    S = summaries.shape[1]
    cand, summ = (B, Cn, d), (B, S, d)
    _shaped(candidates, (("candidates", candidates, cand), ("summaries", summaries, summ), ("d_out", d_out, cand),
                         ("d_candidates", d_candidates, cand), ("d_summaries", d_summaries, summ)))
    desc = AttendDesc(B=B, C=Cn, S=S, d=d, H=H, dtype=_dtype_code(candidates), scale=scale,
                      flags=VISTA_FLAG_SELF_TERM if self_term else 0)
    workspace = _workspace(workspace, lambda: lib().vista_target_attend_backward_workspace_bytes(C.byref(desc)), candidates)
    st = lib().vista_target_attend_backward(C.byref(desc), candidates.data_ptr(), summaries.data_ptr(), d_out.data_ptr(),
                                            d_candidates.data_ptr(), d_summaries.data_ptr(), _dev(workspace, "workspace"),
                                            workspace.numel(), _stream())
    if st != VISTA_OK:
        raise VistaError(st)
    return workspace


def vista_quantize_summaries(y, codes, scales, *, H):
    """Cache codec: y [..., d] -> codes int8 [..., d], scales float32 [..., H] (device tensors)."""
    d = y.shape[-1]
    desc = CodecDesc(rows=y.numel() // d, d=d, H=H, dtype=_dtype_code(y))
    if codes.dtype != torch.int8 or scales.dtype != torch.float32:
        raise TypeError("codes must be int8 and scales float32")
    st = lib().vista_quantize_summaries(C.byref(desc), _dev(y, "y"), _dev(codes, "codes"), _dev(scales, "scales"),
                                        _stream())
    if st != VISTA_OK:
        raise VistaError(st)


def vista_target_attend_q8(candidates, codes, scales, out, *, H, scale=0.0, self_term=False):
    """Stage 2 on quantized summaries: codes int8 [B,S,d], scales float32 [B,S,H]."""
    B, Cn, d = candidates.shape
    S = codes.shape[1]
    desc = AttendDesc(B=B, C=Cn, S=S, d=d, H=H, dtype=_dtype_code(candidates), scale=scale,
                      flags=VISTA_FLAG_SELF_TERM if self_term else 0)
    if codes.dtype != torch.int8 or scales.dtype != torch.float32:
        raise TypeError("codes must be int8 and scales float32")
    st = lib().vista_target_attend_q8(C.byref(desc), _dev(candidates, "candidates"), _dev(codes, "codes"),
                                      _dev(scales, "scales"), _dev(out, "out"), _stream())
    if st != VISTA_OK:
        raise VistaError(st)


def vista_summarize_static(history_emb, offsets, virtual_queries, W_k, W_v, out, *, H, scale=0.0,
                           segment_items=0, offsets_host=None, attn=VISTA_ATTN_SOFTMAX, self_term=False):
    """Stage 1 on the library's static scratch: no workspace argument, nothing allocated."""
    B = offsets.numel() - 1
    S, d = virtual_queries.shape[-2:]
    N = history_emb.shape[0]
    desc = summarize_desc(B, S, d, H, _dtype_code(history_emb), N, virtual_queries.dim() == 3, scale,
                          segment_items, attn, self_term)
    host = None
    if offsets_host is not None:
        if offsets_host.is_cuda or offsets_host.dtype != torch.int64:
            raise ValueError("offsets_host must be a CPU int64 tensor")
        host = offsets_host.contiguous().data_ptr()
    if offsets.dtype != torch.int64:
        raise TypeError("offsets must be int64")
    st = lib().vista_summarize_static(C.byref(desc), _dev(history_emb, "history_emb") if N else None,
                                      _dev(offsets, "offsets"), host, _dev(virtual_queries, "virtual_queries"),
                                      _dev(W_k, "W_k"), _dev(W_v, "W_v"), _dev(out, "out"), _stream())
    if st != VISTA_OK:
        raise VistaError(st)


def vista_target_attend(candidates, summaries, out, *, H, scale=0.0, self_term=False):
    """Stage 2.  candidates [B,C,d], summaries [B,S,d], out [B,C,d]; device, same dtype."""
    B, Cn, d = candidates.shape
    S = summaries.shape[1]
    desc = AttendDesc(B=B, C=Cn, S=S, d=d, H=H, dtype=_dtype_code(candidates), scale=scale,
                      flags=VISTA_FLAG_SELF_TERM if self_term else 0)
    st = lib().vista_target_attend(C.byref(desc), _dev(candidates, "candidates"),
                                   _dev(summaries, "summaries"), _dev(out, "out"), _stream())
    if st != VISTA_OK:
        raise VistaError(st)


def vista_sglu_ffn(y, W_g, W_u, W_o, out, *, eps=0.0):
    """Gated block between layers.  y [rows,d] (any leading shape), W_g/W_u [d,d_ff], W_o [d_ff,d]."""
    d = y.shape[-1]
    rows = y.numel() // d
    desc = FfnDesc(rows=rows, d=d, d_ff=W_g.shape[1], dtype=_dtype_code(y), eps=eps)
    st = lib().vista_sglu_ffn(C.byref(desc), _dev(y, "y"), _dev(W_g, "W_g"), _dev(W_u, "W_u"),
                              _dev(W_o, "W_o"), _dev(out, "out"), _stream())
    if st != VISTA_OK:
        raise VistaError(st)


def _norm_desc(x: torch.Tensor, eps: float) -> NormDesc:
    d = x.shape[-1]
    return NormDesc(x.numel() // d if d else 0, d, _dtype_code(x), eps)


def vista_layer_norm(x, weight, bias, y, *, eps=0.0):
    """Layer norm of the rows of x [..., d] into y (which may be x); weight and bias [d], each may be None."""
    desc = _norm_desc(x, eps)
    row = (desc.d,)
    _shaped(x, (("x", x, x.shape), ("weight", weight, row), ("bias", bias, row), ("y", y, x.shape)))
    st = lib().vista_layer_norm(C.byref(desc), x.data_ptr(), _at(weight), _at(bias), y.data_ptr(), _stream())
    if st != VISTA_OK:
        raise VistaError(st)


def vista_layer_norm_backward(x, weight, d_y, d_x, d_weight, d_bias, *, eps=0.0, workspace=None):
    """Gradients of layer norm: d_y [..., d] -> d_x (which may be d_y), d_weight and d_bias [d] (each may be None).  Returns
    the workspace, which may be passed to the next call; None where neither sum is wanted."""
    desc = _norm_desc(x, eps)
    row = (desc.d,)
    _shaped(x, (("x", x, x.shape), ("weight", weight, row), ("d_y", d_y, x.shape), ("d_x", d_x, x.shape),
                ("d_weight", d_weight, row), ("d_bias", d_bias, row)))
    if d_weight is not None or d_bias is not None:
        workspace = _workspace(workspace, lambda: lib().vista_layer_norm_backward_workspace_bytes(C.byref(desc)), x)
    st = lib().vista_layer_norm_backward(C.byref(desc), x.data_ptr(), _at(weight), d_y.data_ptr(), d_x.data_ptr(), _at(d_weight),
                                         _at(d_bias), None if workspace is None else _dev(workspace, "workspace"),
                                         0 if workspace is None else workspace.numel(), _stream())
    if st != VISTA_OK:
        raise VistaError(st)
    return workspace
