"""Thin Python binding of libhatq (ctypes).

Argument marshalling only: every step of the operator runs in the library's HIP
kernels.  PyTorch supplies device memory (tensors passed by ``data_ptr()``) and
the stream (``torch.cuda.current_stream()``).  There is no fallback: if the
library is missing or cannot be loaded, every call raises.

The function names mirror the C ABI in ``include/hatq.h``.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import Optional, Tuple

import torch

from . import build as _build

HATQ_OK, HATQ_EINVAL, HATQ_EUNSUPPORTED, HATQ_EWORKSPACE, HATQ_EHIP = range(5)
HATQ_DH, HATQ_WH = 0, 1
HATQ_OUT_I32, HATQ_OUT_F32, HATQ_OUT_I8 = 0, 1, 2
HATQ_PAIRED, HATQ_XQ_C64, HATQ_YQ_C64 = 1, 2, 4
FORMS = {"DH": HATQ_DH, "WH": HATQ_WH}


class HatqError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


class ConvDesc(ctypes.Structure):
    _fields_ = [("cin", ctypes.c_int32), ("cout", ctypes.c_int32), ("k", ctypes.c_int32),
                ("stride", ctypes.c_int32), ("pad", ctypes.c_int32), ("out_pad", ctypes.c_int32),
                ("transposed", ctypes.c_int32), ("hblock", ctypes.c_int32)]


class Weights(ctypes.Structure):
    _fields_ = [("d", ConvDesc), ("form", ctypes.c_int32), ("cin_pad", ctypes.c_int32),
                ("cout_pad", ctypes.c_int32), ("k_total", ctypes.c_int32),
                ("k_stride", ctypes.c_int32), ("wq", ctypes.c_void_p),
                ("w_scale", ctypes.c_void_p), ("bias", ctypes.c_void_p),
                ("wpack", ctypes.c_void_p), ("pack_stride", ctypes.c_int32)]


class LinearWeights(ctypes.Structure):
    _fields_ = [("experts", ctypes.c_int32), ("cin", ctypes.c_int32), ("cout", ctypes.c_int32),
                ("gated", ctypes.c_int32), ("hblock", ctypes.c_int32), ("k_stride", ctypes.c_int32),
                ("cout_pad", ctypes.c_int32), ("wpack", ctypes.c_void_p), ("w_scale", ctypes.c_void_p),
                ("bias", ctypes.c_void_p)]


class Linear4Weights(ctypes.Structure):
    _fields_ = [("cin", ctypes.c_int32), ("cout", ctypes.c_int32), ("gated", ctypes.c_int32),
                ("hblock", ctypes.c_int32), ("group", ctypes.c_int32), ("k_stride", ctypes.c_int32),
                ("cout_pad", ctypes.c_int32), ("wpack", ctypes.c_void_p), ("w_scale", ctypes.c_void_p),
                ("bias", ctypes.c_void_p)]


class Cache4View(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("dim", ctypes.c_int32), ("hblock", ctypes.c_int32), ("buf", ctypes.c_void_p)]


class Heads(ctypes.Structure):
    _fields_ = [("type", ctypes.c_int32), ("row_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("p", ctypes.c_void_p)]


EXPORTS = ["hatq_status_string", "hatq_conv_out_hw", "hatq_weights_bytes", "hatq_prepare_weights",
           "hatq_export_weights", "hatq_pack_weights", "hatq_fwht_quant_ws_bytes", "hatq_fwht_quant_act",
           "hatq_fwht_quant_act_noalloc", "hatq_fwht_quant_act_c64", "hatq_conv_int8",
           "hatq_conv_int8_requant", "hatq_int_table_len", "hatq_int_transition_params",
           "hatq_conv_int8_int_transition", "hatq_range_expansion", "hatq_select_form", "hatq_hadamard_order",
           "hatq_fwht_quant_affine_ws_bytes", "hatq_fwht_quant_act_affine", "hatq_tapsum_len",
           "hatq_weight_tapsums", "hatq_conv_int8_affine",
           "hatq_layer_ws_bytes", "hatq_layer_forward",
           "hatq_linear_weights_bytes", "hatq_prepare_linear", "hatq_pack_linear", "hatq_token_quant",
           "hatq_linear_int8", "hatq_linear_ws_bytes", "hatq_linear_forward", "hatq_experts_int8",
           "hatq_experts_forward", "hatq_expert_order_ws_bytes", "hatq_expert_order", "hatq_expert_combine",
           "hatq_expert_mlp_ws_bytes", "hatq_expert_mlp",
           "hatq_linear4_weights_bytes", "hatq_prepare_linear4", "hatq_pack_linear4", "hatq_linear4_ws_bytes",
           "hatq_linear4_forward", "hatq_cache4_bytes", "hatq_cache4_init", "hatq_cache4_append", "hatq_cache4_read",
           "hatq_attention4_ws_bytes", "hatq_attention4"]

_lib = None


def lib_path() -> str:
    return _build.LIB


def load(build_if_missing: bool = False):
    """Load libhatq.so; raise if it is absent (no silent fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    path = lib_path()
    if not os.path.exists(path):
        if not build_if_missing:
            raise RuntimeError(f"libhatq.so not built ({path}); run __graft_entry__.build()")
        _build.build()
    L = ctypes.CDLL(path)
    P, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    L.hatq_status_string.argtypes = [i32]
    L.hatq_status_string.restype = ctypes.c_char_p
    L.hatq_conv_out_hw.argtypes = [ctypes.POINTER(ConvDesc), i32, i32, ctypes.POINTER(i32), ctypes.POINTER(i32)]
    L.hatq_conv_out_hw.restype = i32
    L.hatq_weights_bytes.argtypes = [ctypes.POINTER(ConvDesc), i32]
    L.hatq_weights_bytes.restype = sz
    L.hatq_prepare_weights.argtypes = [ctypes.POINTER(ConvDesc), i32, P, P, P, sz, ctypes.POINTER(Weights), P]
    L.hatq_prepare_weights.restype = i32
    L.hatq_export_weights.argtypes = [ctypes.POINTER(Weights), P, P, P, P]
    L.hatq_export_weights.restype = i32
    L.hatq_pack_weights.argtypes = [ctypes.POINTER(Weights), P]
    L.hatq_pack_weights.restype = i32
    L.hatq_fwht_quant_ws_bytes.argtypes = [i32]
    L.hatq_fwht_quant_ws_bytes.restype = sz
    L.hatq_fwht_quant_act.argtypes = [P, i32, i32, i32, i32, i32, P, P, P, P, sz, P]
    L.hatq_fwht_quant_act.restype = i32
    L.hatq_fwht_quant_act_noalloc.argtypes = [P, i32, i32, i32, i32, i32, P, P, P]
    L.hatq_fwht_quant_act_noalloc.restype = i32
    L.hatq_fwht_quant_act_c64.argtypes = [P, i32, i32, i32, i32, i32, P, P, P, P, sz, P]
    L.hatq_fwht_quant_act_c64.restype = i32
    L.hatq_conv_int8.argtypes = [ctypes.POINTER(Weights), P, P, i32, i32, i32, i32, P, P, i32, P, i32, P]
    L.hatq_conv_int8.restype = i32
    L.hatq_conv_int8_requant.argtypes = [ctypes.POINTER(Weights), P, P, i32, i32, i32, i32, P, P, P, i32, P]
    L.hatq_conv_int8_requant.restype = i32
    L.hatq_int_table_len.argtypes = [ctypes.POINTER(Weights)]
    L.hatq_int_table_len.restype = sz
    L.hatq_int_transition_params.argtypes = [ctypes.POINTER(Weights), ctypes.c_float, ctypes.c_float, i32, P, P]
    L.hatq_int_transition_params.restype = i32
    L.hatq_conv_int8_int_transition.argtypes = [ctypes.POINTER(Weights), P, i32, i32, i32, i32, P, P, i32, P]
    L.hatq_conv_int8_int_transition.restype = i32
    L.hatq_range_expansion.argtypes = [P, i32, i32, i32, i32, i32, P, P, P, P]
    L.hatq_fwht_quant_affine_ws_bytes.argtypes = [i32]
    L.hatq_fwht_quant_affine_ws_bytes.restype = sz
    L.hatq_fwht_quant_act_affine.argtypes = [P, i32, i32, i32, i32, i32, P, P, P, P, sz, P]
    L.hatq_fwht_quant_act_affine.restype = i32
    L.hatq_tapsum_len.argtypes = [ctypes.POINTER(Weights)]
    L.hatq_tapsum_len.restype = sz
    L.hatq_weight_tapsums.argtypes = [ctypes.POINTER(Weights), P, P]
    L.hatq_weight_tapsums.restype = i32
    L.hatq_conv_int8_affine.argtypes = [ctypes.POINTER(Weights), P, P, P, P, i32, i32, i32, i32, P, P]
    L.hatq_conv_int8_affine.restype = i32
    L.hatq_range_expansion.restype = i32
    L.hatq_select_form.argtypes = [ctypes.c_int64, ctypes.c_int64, ctypes.c_double, ctypes.POINTER(i32)]
    L.hatq_select_form.restype = i32
    L.hatq_hadamard_order.argtypes = [i32]
    L.hatq_hadamard_order.restype = i32
    L.hatq_layer_ws_bytes.argtypes = [ctypes.POINTER(Weights), i32, i32, i32]
    L.hatq_layer_ws_bytes.restype = sz
    L.hatq_layer_forward.argtypes = [ctypes.POINTER(Weights), i32, P, i32, i32, i32, P, P, P, i32, P, P,
                                     sz, P]
    L.hatq_layer_forward.restype = i32
    i64, W = ctypes.c_int64, ctypes.POINTER(LinearWeights)
    L.hatq_linear_weights_bytes.argtypes = [i32] * 5
    L.hatq_linear_weights_bytes.restype = sz
    L.hatq_prepare_linear.argtypes = [i32] * 5 + [P, i32, P, P, sz, W, P]
    L.hatq_prepare_linear.restype = i32
    L.hatq_pack_linear.argtypes = [i32] * 5 + [P, P, P, P, sz, W, P]
    L.hatq_pack_linear.restype = i32
    L.hatq_token_quant.argtypes = [P, i32, i32, i32, i64, i32, P, P, P]
    L.hatq_token_quant.restype = i32
    L.hatq_linear_int8.argtypes = [W, P, P, i32, P, i32, i64, P]
    L.hatq_linear_int8.restype = i32
    L.hatq_linear_ws_bytes.argtypes = [W, i32]
    L.hatq_linear_ws_bytes.restype = sz
    L.hatq_linear_forward.argtypes = [W, P, i32, i32, i64, P, i32, i64, P, sz, P]
    L.hatq_linear_forward.restype = i32
    L.hatq_experts_int8.argtypes = [W, P, P, i32, P, P, i32, P, i32, i64, P]
    L.hatq_experts_int8.restype = i32
    L.hatq_experts_forward.argtypes = [W, P, i32, i32, i64, P, P, i32, P, i32, i64, P, sz, P]
    L.hatq_experts_forward.restype = i32
    L.hatq_expert_order_ws_bytes.argtypes = [i32] * 3
    L.hatq_expert_order_ws_bytes.restype = sz
    L.hatq_expert_order.argtypes = [P, i32, i32, i32, P, P, P, P, sz, P]
    L.hatq_expert_order.restype = i32
    L.hatq_expert_combine.argtypes = [P, i32, i32, i64, P, P, i32, i32, P, i32, i64, P]
    L.hatq_expert_combine.restype = i32
    L.hatq_expert_mlp_ws_bytes.argtypes = [W, W, i32, i32]
    L.hatq_expert_mlp_ws_bytes.restype = sz
    L.hatq_expert_mlp.argtypes = [W, W, P, i32, i32, i64, P, P, i32, P, i32, i64, P, sz, P]
    L.hatq_expert_mlp.restype = i32
    W4 = ctypes.POINTER(Linear4Weights)
    L.hatq_linear4_weights_bytes.argtypes = [i32] * 5
    L.hatq_linear4_weights_bytes.restype = sz
    L.hatq_prepare_linear4.argtypes = [i32] * 5 + [P, i32, P, P, sz, W4, P]
    L.hatq_prepare_linear4.restype = i32
    L.hatq_pack_linear4.argtypes = [i32] * 5 + [P, P, P, P, sz, W4, P]
    L.hatq_pack_linear4.restype = i32
    L.hatq_linear4_ws_bytes.argtypes = [W4, i32]
    L.hatq_linear4_ws_bytes.restype = sz
    L.hatq_linear4_forward.argtypes = [W4, P, i32, i32, i64, P, i32, i64, P, sz, P]
    L.hatq_linear4_forward.restype = i32
    C, H, f32 = ctypes.POINTER(Cache4View), ctypes.POINTER(Heads), ctypes.c_float
    L.hatq_cache4_bytes.argtypes = [i32] * 5
    L.hatq_cache4_bytes.restype = sz
    L.hatq_cache4_init.argtypes = [i32, i32, i32, i32, i32, P, sz, C]
    L.hatq_cache4_init.restype = i32
    for f in (L.hatq_cache4_append, L.hatq_cache4_read):
        f.argtypes = [C, H, H, i32, P, i32, P, P, i32, P]
        f.restype = i32
    L.hatq_attention4_ws_bytes.argtypes = [C] + [i32] * 7
    L.hatq_attention4_ws_bytes.restype = sz
    L.hatq_attention4.argtypes = [C, H, H, i32, i32, P, i32, P, P, i32, f32, i32, i32, i32, P, sz, P]
    L.hatq_attention4.restype = i32
    _lib = L
    return L


def status_string(s: int) -> str:
    return load().hatq_status_string(int(s)).decode()


def _check(status: int, where: str):
    if status != HATQ_OK:
        raise HatqError(status, where)


# The calls of a small layer are bound by this module: a 512x768 stack step was
# 113 us of host time for about 105 us of GPU work.  So each tensor is checked once
# (_need, _nhwc), addresses go to ctypes as plain integers, sizes are formed here
# rather than by another library call, and sizes of buffers that the caller has
# brought are left to the library's own check.
def _ptr(t: Optional[torch.Tensor]):
    """The address of a tensor that _need or _nhwc has checked, or None."""
    return None if t is None else t.data_ptr()


def _need(t: Optional[torch.Tensor], name: str, dtype: torch.dtype, numel: int, optional: bool = False):
    """Raise ValueError unless t is a contiguous device tensor of `dtype` with at
    least `numel` elements (the library trusts the pointers it is given)."""
    if t is not None and t.is_cuda and t.dtype is dtype and t.is_contiguous() and t.numel() >= numel:
        return
    if t is None:
        if optional:
            return
        raise ValueError(f"{name}: tensor required")
    if not t.is_cuda:
        raise ValueError(f"{name}: device tensor expected")
    if t.dtype != dtype:
        raise ValueError(f"{name}: {dtype} expected, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: contiguous tensor expected")
    if t.numel() < numel:
        raise ValueError(f"{name}: {numel} elements needed, got {t.numel()}")


def _nhwc(t: torch.Tensor, name: str, dtype: torch.dtype, channels: Optional[int] = None):
    shape = t.shape
    if len(shape) != 4:
        raise ValueError(f"{name}: NHWC tensor expected, got shape {tuple(shape)}")
    if channels is not None and shape[3] != channels:
        raise ValueError(f"{name}: {channels} channels expected, got {shape[3]}")
    _need(t, name, dtype, 0)
    return shape


# (a private name of torch: where a version lacks it, the public call, 1-2 us slower)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream=None):
    """The raw stream handle: the given stream's, or that of the current stream of
    the current device."""
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def desc(cin, cout, k, stride, pad, hblock, transposed=False, out_pad=0) -> ConvDesc:
    return ConvDesc(int(cin), int(cout), int(k), int(stride), int(pad), int(out_pad),
                    int(bool(transposed)), int(hblock))


def hatq_conv_out_hw(d: ConvDesc, h: int, w: int) -> Tuple[int, int]:
    ho, wo = ctypes.c_int32(), ctypes.c_int32()
    _check(load().hatq_conv_out_hw(ctypes.byref(d), h, w, ctypes.byref(ho), ctypes.byref(wo)),
           "hatq_conv_out_hw")
    return ho.value, wo.value


def _out_hw(d: ConvDesc, h: int, w: int) -> Tuple[int, int]:
    """hatq_conv_out_hw's sizes without the call (which reports what is invalid)."""
    k, st, p2 = d.k, d.stride, 2 * d.pad
    if d.transposed:
        op = d.out_pad
        ho, wo = (h - 1) * st - p2 + k + op, (w - 1) * st - p2 + k + op
    else:
        if st <= 0 or h + p2 < k or w + p2 < k:
            return hatq_conv_out_hw(d, h, w)
        ho, wo = (h + p2 - k) // st + 1, (w + p2 - k) // st + 1
    if not (0 < ho < 2 ** 31 and 0 < wo < 2 ** 31 and h > 0 and w > 0):
        return hatq_conv_out_hw(d, h, w)
    return ho, wo


def hatq_weights_bytes(d: ConvDesc, form) -> int:
    return int(load().hatq_weights_bytes(ctypes.byref(d), FORMS.get(form, form)))


@dataclass
class PreparedLayer:
    """Prepared weights of one layer: the device buffer and the C view into it."""
    buf: torch.Tensor
    w: Weights
    form: int

    @property
    def cout_pad(self) -> int:
        return self.w.cout_pad

    @property
    def cin_pad(self) -> int:
        return self.w.cin_pad

    @property
    def k_stride(self) -> int:
        return self.w.k_stride

    def wq(self) -> torch.Tensor:
        """int8 [cout_pad, k_stride] view of the packed codes."""
        n = self.w.cout_pad * self.w.k_stride
        return self.buf[:n].view(self.w.cout_pad, self.w.k_stride)

    def w_scale(self) -> torch.Tensor:
        off = self.w.w_scale - self.buf.data_ptr()
        return self.buf[off:off + 4 * self.w.cout_pad].view(torch.float32)

    def bias(self) -> torch.Tensor:
        off = self.w.bias - self.buf.data_ptr()
        return self.buf[off:off + 4 * self.w.cout_pad].view(torch.float32)

    def wpack(self) -> torch.Tensor:
        """int8 [pack_stride/64, cout_pad, 64] view of the kernel-order copy."""
        off = self.w.wpack - self.buf.data_ptr()
        n = self.w.cout_pad * self.w.pack_stride
        return self.buf[off:off + n].view(self.w.pack_stride // 64, self.w.cout_pad, 64)


def hatq_prepare_weights(d: ConvDesc, form, w: torch.Tensor, bias: Optional[torch.Tensor] = None,
                         stream=None) -> PreparedLayer:
    f = FORMS.get(form, form)
    nbytes = hatq_weights_bytes(d, f)
    if nbytes == 0:
        raise HatqError(HATQ_EINVAL, "hatq_weights_bytes")
    buf = torch.zeros(nbytes, dtype=torch.int8, device=w.device)
    out = Weights()
    w = w.contiguous().float()
    b = None if bias is None else bias.contiguous().float()
    _need(w, "w", torch.float32, d.cout * d.cin * d.k * d.k)
    _need(b, "bias", torch.float32, d.cout, optional=True)
    _check(load().hatq_prepare_weights(ctypes.byref(d), f, _ptr(w), _ptr(b), _ptr(buf), nbytes,
                                       ctypes.byref(out), _stream(stream)), "hatq_prepare_weights")
    return PreparedLayer(buf, out, f)


def hatq_export_weights(layer: PreparedLayer, stream=None):
    """Host copies of the prepared operator: (codes int8 [cout_pad, k, k, cin_pad],
    w_scale fp32 [cout_pad], bias fp32 [cout_pad]); waits for the stream."""
    k, cp, co = layer.w.d.k, layer.w.cin_pad, layer.w.cout_pad
    wq = torch.empty((co, k, k, cp), dtype=torch.int8, pin_memory=True)
    sc = torch.empty(co, dtype=torch.float32, pin_memory=True)
    b = torch.empty(co, dtype=torch.float32, pin_memory=True)
    s = stream if stream is not None else torch.cuda.current_stream()
    _check(load().hatq_export_weights(ctypes.byref(layer.w), ctypes.c_void_p(wq.data_ptr()),
                                      ctypes.c_void_p(sc.data_ptr()), ctypes.c_void_p(b.data_ptr()), _stream(s)),
           "hatq_export_weights")
    s.synchronize()
    return wq, sc, b


def hatq_pack_weights(layer: PreparedLayer, stream=None) -> None:
    """Rebuild the kernel-order copy after codes were written into ``layer.wq()``."""
    _check(load().hatq_pack_weights(ctypes.byref(layer.w), _stream(stream)), "hatq_pack_weights")


def hatq_fwht_quant_act(x: torch.Tensor, hblock: int, absmax: Optional[torch.Tensor] = None,
                        xq: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                        ws: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """x fp32 NHWC -> (int8 codes NHWC, per-sample scale fp32 [n]).  Output and
    workspace tensors may be passed in to avoid allocation."""
    n, h, w, c = _nhwc(x, "x", torch.float32)
    if xq is None:
        xq = torch.empty((n, h, w, c), dtype=torch.int8, device=x.device)
    sc = scale if scale is not None else torch.empty(n, dtype=torch.float32, device=x.device)
    _need(xq, "xq", torch.int8, x.numel())
    _need(sc, "scale", torch.float32, n)
    _need(absmax, "absmax", torch.float32, n, optional=True)
    if ws is None:
        ws = torch.empty(max(int(load().hatq_fwht_quant_ws_bytes(n)), 4), dtype=torch.int8, device=x.device)
    _need(ws, "ws", torch.int8, 0)
    _check(load().hatq_fwht_quant_act(_ptr(x), n, h, w, c, int(hblock), _ptr(absmax), _ptr(xq), _ptr(sc),
                                      _ptr(ws), ws.numel(), _stream(stream)), "hatq_fwht_quant_act")
    return xq, sc


HATQ_NOALLOC_MAX_SAMPLES = 4096


def hatq_fwht_quant_act_noalloc(x: torch.Tensor, hblock: int, xq: torch.Tensor, scale: torch.Tensor,
                                stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """hatq_fwht_quant_act (two passes) with the library's static scratch: the
    caller passes the outputs; nothing is allocated."""
    n, h, w, c = _nhwc(x, "x", torch.float32)
    _need(xq, "xq", torch.int8, x.numel())
    _need(scale, "scale", torch.float32, n)
    _check(load().hatq_fwht_quant_act_noalloc(_ptr(x), n, h, w, c, int(hblock), _ptr(xq), _ptr(scale),
                                              _stream(stream)), "hatq_fwht_quant_act_noalloc")
    return xq, scale


def hatq_fwht_quant_act_c64(x: torch.Tensor, hblock: int, absmax: Optional[torch.Tensor] = None,
                            xq: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                            ws: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """hatq_fwht_quant_act with the codes chunk-major: int8 [n, c/64, h, w, 64]."""
    n, h, w, c = _nhwc(x, "x", torch.float32)
    if c % 64:
        raise HatqError(HATQ_EUNSUPPORTED, "hatq_fwht_quant_act_c64 (c % 64)")
    if xq is None:
        xq = torch.empty((n, c // 64, h, w, 64), dtype=torch.int8, device=x.device)
    sc = scale if scale is not None else torch.empty(n, dtype=torch.float32, device=x.device)
    _need(xq, "xq", torch.int8, x.numel())
    _need(sc, "scale", torch.float32, n)
    _need(absmax, "absmax", torch.float32, n, optional=True)
    if ws is None:
        ws = torch.empty(max(int(load().hatq_fwht_quant_ws_bytes(n)), 4), dtype=torch.int8, device=x.device)
    _need(ws, "ws", torch.int8, 0)
    _check(load().hatq_fwht_quant_act_c64(_ptr(x), n, h, w, c, int(hblock), _ptr(absmax), _ptr(xq), _ptr(sc),
                                          _ptr(ws), ws.numel(), _stream(stream)), "hatq_fwht_quant_act_c64")
    return xq, sc


def to_c64(q: torch.Tensor) -> torch.Tensor:
    """NHWC codes [n, h, w, c] -> chunk-major [n, c/64, h, w, 64] (a copy)."""
    n, h, w, c = q.shape
    return q.view(n, h, w, c // 64, 64).permute(0, 3, 1, 2, 4).contiguous()


def from_c64(q: torch.Tensor) -> torch.Tensor:
    """Chunk-major codes [n, c/64, h, w, 64] -> NHWC [n, h, w, c] (a copy)."""
    n, m, h, w, _ = q.shape
    return q.permute(0, 2, 3, 1, 4).reshape(n, h, w, m * 64).contiguous()


def _codes_in(xq: torch.Tensor, cin_pad: int):
    """(n, h, w, flag) of a layer's input codes: NHWC [n, h, w, cin_pad], or
    chunk-major [n, cin_pad/64, h, w, 64] (HATQ_XQ_C64)."""
    if xq.dim() == 5:
        n, m, h, w, c64 = xq.shape
        if m * 64 != cin_pad or c64 != 64:
            raise ValueError(f"xq: chunk-major shape {tuple(xq.shape)} for cin_pad {cin_pad}")
        _need(xq, "xq", torch.int8, n * h * w * cin_pad)
        return n, h, w, HATQ_XQ_C64
    n, h, w, _ = _nhwc(xq, "xq", torch.int8, cin_pad)
    return n, h, w, 0


def _codes_out_shape(n: int, ho: int, wo: int, c: int, c64: bool):
    return (n, c // 64, ho, wo, 64) if c64 else (n, ho, wo, c)


def _flags(paired: bool) -> int:
    return HATQ_PAIRED if paired else 0


def hatq_conv_int8(layer: PreparedLayer, xq: torch.Tensor, act_scale: torch.Tensor, out_mode=HATQ_OUT_F32,
                   next_hblock: int = 0, next_absmax: Optional[torch.Tensor] = None, y=None, stream=None,
                   absmax_only: bool = False, out_scale: Optional[torch.Tensor] = None, paired: bool = False,
                   yq_c64: bool = False):
    """absmax_only: F32 mode with y = NULL, producing next_absmax alone (returns None).
    out_mode HATQ_OUT_I8: y receives the next operand's codes with the static
    per-sample scale out_scale (chunk-major with yq_c64).  paired: the
    HATQ_PAIRED flag.  A 5-d xq is chunk-major (HATQ_XQ_C64)."""
    n, h, w, xf = _codes_in(xq, layer.w.cin_pad)
    fl = _flags(paired) | xf | (HATQ_YQ_C64 if yq_c64 else 0)
    _need(act_scale, "act_scale", torch.float32, n)
    _need(next_absmax, "next_absmax", torch.float32, n, optional=True)
    _need(out_scale, "out_scale", torch.float32, n, optional=True)
    ho, wo = _out_hw(layer.w.d, h, w)
    if absmax_only:
        _check(load().hatq_conv_int8(ctypes.byref(layer.w), _ptr(xq), _ptr(act_scale), n, h, w, int(out_mode),
                                     _ptr(out_scale), None, int(next_hblock), _ptr(next_absmax), fl,
                                     _stream(stream)),
               "hatq_conv_int8")
        return None
    if out_mode == HATQ_OUT_I32:
        shape, dt = (n, ho, wo, layer.w.cout_pad), torch.int32
    elif out_mode == HATQ_OUT_I8:
        shape, dt = _codes_out_shape(n, ho, wo, layer.w.d.cout, yq_c64), torch.int8
    else:
        shape, dt = (n, ho, wo, layer.w.d.cout), torch.float32
    if y is None:
        y = torch.empty(shape, dtype=dt, device=xq.device)
    _need(y, "y", dt, n * ho * wo * (layer.w.cout_pad if out_mode == HATQ_OUT_I32 else layer.w.d.cout))
    _check(load().hatq_conv_int8(ctypes.byref(layer.w), _ptr(xq), _ptr(act_scale), n, h, w, int(out_mode),
                                 _ptr(out_scale), _ptr(y), int(next_hblock), _ptr(next_absmax), fl,
                                 _stream(stream)),
           "hatq_conv_int8")
    return y


def hatq_conv_int8_requant(layer: PreparedLayer, xq: torch.Tensor, act_scale: torch.Tensor, next_hblock: int,
                           next_absmax: Optional[torch.Tensor] = None, next_scale: Optional[torch.Tensor] = None,
                           yq: Optional[torch.Tensor] = None, stream=None, paired: bool = False,
                           yq_c64: bool = False):
    """Conv with the requantizing epilogue: returns (yq, next_scale), the next
    layer's codes (chunk-major with yq_c64) and scale.  A 5-d xq is chunk-major."""
    n, h, w, xf = _codes_in(xq, layer.w.cin_pad)
    _need(act_scale, "act_scale", torch.float32, n)
    _need(next_absmax, "next_absmax", torch.float32, n, optional=True)
    ho, wo = _out_hw(layer.w.d, h, w)
    if yq is None:
        yq = torch.empty(_codes_out_shape(n, ho, wo, layer.w.d.cout, yq_c64), dtype=torch.int8, device=xq.device)
    if next_scale is None:
        next_scale = torch.empty((n,), dtype=torch.float32, device=xq.device)
    _need(yq, "yq", torch.int8, n * ho * wo * layer.w.d.cout)
    _need(next_scale, "next_scale", torch.float32, n)
    _check(load().hatq_conv_int8_requant(ctypes.byref(layer.w), _ptr(xq), _ptr(act_scale), n, h, w,
                                         int(next_hblock), _ptr(next_absmax), _ptr(next_scale), _ptr(yq),
                                         _flags(paired) | xf | (HATQ_YQ_C64 if yq_c64 else 0), _stream(stream)),
           "hatq_conv_int8_requant")
    return yq, next_scale


def hatq_int_table_len(layer: PreparedLayer) -> int:
    return int(load().hatq_int_table_len(ctypes.byref(layer.w)))


def hatq_int_transition_params(layer: PreparedLayer, s_x: float, s_y: float, next_hblock: int,
                               table: Optional[torch.Tensor] = None, device="cuda", stream=None):
    """Integer transition table (M, b_int, shift) from static scales: returns
    (table, shift).  The library call does not wait; this wrapper reads the shift
    back (-1: none fits, then the call is reported as HATQ_EUNSUPPORTED here)."""
    if table is None:
        table = torch.empty((hatq_int_table_len(layer),), dtype=torch.int32, device=device)
    _need(table, "table", torch.int32, hatq_int_table_len(layer))
    _check(load().hatq_int_transition_params(ctypes.byref(layer.w), float(s_x), float(s_y), int(next_hblock),
                                             _ptr(table), _stream(stream)),
           "hatq_int_transition_params")
    shift = int(table[2 * layer.w.cout_pad].item())
    if shift < 0:
        raise HatqError(HATQ_EUNSUPPORTED, "hatq_int_transition_params (no shift fits)")
    return table, shift


def hatq_conv_int8_int_transition(layer: PreparedLayer, xq: torch.Tensor, next_hblock: int, table: torch.Tensor,
                                  yq: Optional[torch.Tensor] = None, stream=None, paired: bool = False,
                                  yq_c64: bool = False) -> torch.Tensor:
    """Conv with the integer-only epilogue: the next layer's codes (chunk-major
    with yq_c64).  A 5-d xq is chunk-major."""
    n, h, w, xf = _codes_in(xq, layer.w.cin_pad)
    _need(table, "table", torch.int32, hatq_int_table_len(layer))
    ho, wo = _out_hw(layer.w.d, h, w)
    if yq is None:
        yq = torch.empty(_codes_out_shape(n, ho, wo, layer.w.d.cout, yq_c64), dtype=torch.int8, device=xq.device)
    _need(yq, "yq", torch.int8, n * ho * wo * layer.w.d.cout)
    _check(load().hatq_conv_int8_int_transition(ctypes.byref(layer.w), _ptr(xq), n, h, w, int(next_hblock),
                                                _ptr(table), _ptr(yq), _flags(paired) | xf |
                                                (HATQ_YQ_C64 if yq_c64 else 0), _stream(stream)),
           "hatq_conv_int8_int_transition")
    return yq


def hatq_fwht_quant_act_affine(x: torch.Tensor, hblock: int, xq: Optional[torch.Tensor] = None,
                               scale: Optional[torch.Tensor] = None, zero: Optional[torch.Tensor] = None,
                               ws: Optional[torch.Tensor] = None, stream=None):
    """x fp32 NHWC -> (int8 codes, per-sample scale fp32 [n], zero point int32 [n])."""
    n, h, w, c = _nhwc(x, "x", torch.float32)
    if xq is None:
        xq = torch.empty((n, h, w, c), dtype=torch.int8, device=x.device)
    if scale is None:
        scale = torch.empty(n, dtype=torch.float32, device=x.device)
    if zero is None:
        zero = torch.empty(n, dtype=torch.int32, device=x.device)
    if ws is None:
        ws = torch.empty(int(load().hatq_fwht_quant_affine_ws_bytes(n)), dtype=torch.int8, device=x.device)
    _need(xq, "xq", torch.int8, x.numel())
    _need(scale, "scale", torch.float32, n)
    _need(zero, "zero", torch.int32, n)
    _need(ws, "ws", torch.int8, 0)
    _check(load().hatq_fwht_quant_act_affine(_ptr(x), n, h, w, c, int(hblock), _ptr(xq), _ptr(scale), _ptr(zero),
                                             _ptr(ws), ws.numel(), _stream(stream)), "hatq_fwht_quant_act_affine")
    return xq, scale, zero


def hatq_weight_tapsums(layer: PreparedLayer, tapsum: Optional[torch.Tensor] = None, device="cuda", stream=None):
    need = int(load().hatq_tapsum_len(ctypes.byref(layer.w)))
    if tapsum is None:
        tapsum = torch.empty(need, dtype=torch.int32, device=device)
    _need(tapsum, "tapsum", torch.int32, need)
    _check(load().hatq_weight_tapsums(ctypes.byref(layer.w), _ptr(tapsum), _stream(stream)), "hatq_weight_tapsums")
    return tapsum


def hatq_conv_int8_affine(layer: PreparedLayer, xq: torch.Tensor, act_scale: torch.Tensor, act_zero: torch.Tensor,
                          tapsum: torch.Tensor, out_mode=HATQ_OUT_F32, y=None, stream=None) -> torch.Tensor:
    n, h, w, _ = _nhwc(xq, "xq", torch.int8, layer.w.cin_pad)
    _need(act_scale, "act_scale", torch.float32, n)
    _need(act_zero, "act_zero", torch.int32, n)
    _need(tapsum, "tapsum", torch.int32, int(load().hatq_tapsum_len(ctypes.byref(layer.w))))
    ho, wo = _out_hw(layer.w.d, h, w)
    if out_mode == HATQ_OUT_I32:
        shape, dt = (n, ho, wo, layer.w.cout_pad), torch.int32
    else:
        shape, dt = (n, ho, wo, layer.w.d.cout), torch.float32
    if y is None:
        y = torch.empty(shape, dtype=dt, device=xq.device)
    _need(y, "y", dt, n * ho * wo * shape[3])
    _check(load().hatq_conv_int8_affine(ctypes.byref(layer.w), _ptr(xq), _ptr(act_scale), _ptr(act_zero),
                                        _ptr(tapsum), n, h, w, int(out_mode), _ptr(y), _stream(stream)),
           "hatq_conv_int8_affine")
    return y


def hatq_range_expansion(x: torch.Tensor, hblock: int, amax: Optional[torch.Tensor] = None,
                         flags: Optional[torch.Tensor] = None, count: Optional[torch.Tensor] = None,
                         stream=None):
    """Per-sample range-expansion indicator of x (fp32 NHWC): returns (amax [2n], flags [n]).
    count, if given, accumulates the number of expanding samples."""
    n, h, w, c = _nhwc(x, "x", torch.float32)
    if amax is None:
        amax = torch.empty(2 * n, dtype=torch.float32, device=x.device)
    if flags is None:
        flags = torch.empty(n, dtype=torch.int32, device=x.device)
    _need(amax, "amax", torch.float32, 2 * n)
    _need(flags, "flags", torch.int32, n)
    _need(count, "count", torch.int32, 1, optional=True)
    _check(load().hatq_range_expansion(_ptr(x), n, h, w, c, int(hblock), _ptr(amax), _ptr(flags), _ptr(count),
                                       _stream(stream)), "hatq_range_expansion")
    return amax, flags


def hatq_select_form(expansions: int, images: int, tau: float = 0.8) -> str:
    f = ctypes.c_int32(-1)
    _check(load().hatq_select_form(int(expansions), int(images), float(tau), ctypes.byref(f)), "hatq_select_form")
    return "WH" if f.value == HATQ_WH else "DH"


def hatq_hadamard_order(c: int) -> int:
    """m(c) of the transform order rule (0: c outside [1, 4096])."""
    return int(load().hatq_hadamard_order(int(c)))


def hatq_layer_ws_bytes(layer: PreparedLayer, n: int, h: int, w: int) -> int:
    return int(load().hatq_layer_ws_bytes(ctypes.byref(layer.w), n, h, w))


def hatq_layer_forward(layer: PreparedLayer, form, x: torch.Tensor, x_absmax: Optional[torch.Tensor] = None,
                       next_hblock: int = 0, next_absmax: Optional[torch.Tensor] = None,
                       act_scale: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None,
                       ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    n, h, w, _ = _nhwc(x, "x", torch.float32, layer.w.d.cin)
    _need(x_absmax, "x_absmax", torch.float32, n, optional=True)
    _need(next_absmax, "next_absmax", torch.float32, n, optional=True)
    _need(act_scale, "act_scale", torch.float32, n, optional=True)
    ho, wo = _out_hw(layer.w.d, h, w)
    if y is None:
        y = torch.empty((n, ho, wo, layer.w.d.cout), dtype=torch.float32, device=x.device)
    _need(y, "y", torch.float32, n * ho * wo * layer.w.d.cout)
    if ws is None:
        ws = torch.empty(max(hatq_layer_ws_bytes(layer, n, h, w), 256), dtype=torch.int8, device=x.device)
    _need(ws, "ws", torch.int8, 0)
    _check(load().hatq_layer_forward(ctypes.byref(layer.w), FORMS.get(form, form), _ptr(x), n, h, w,
                                     _ptr(x_absmax), _ptr(y), _ptr(act_scale), int(next_hblock),
                                     _ptr(next_absmax), _ptr(ws), ws.numel(), _stream(stream)),
           "hatq_layer_forward")
    return y


# ---- linear layers over tokens ------------------------------------------------

# With stream=, a torch.cuda.Stream, a call, what it allocates and the copies it makes of
# its arguments are that stream's, not the current one's: each function calls itself again
# under it.
HATQ_TOKEN_ROWS, HATQ_TOKEN_CODES = 16, 16384
DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


@dataclass
class PreparedLinear:
    """Prepared linear weights: the device buffer and the C view into it."""
    buf: torch.Tensor
    w: LinearWeights
    experts: int
    cin: int
    cout: int
    k_stride: int

    def __post_init__(self):
        self.ref = ctypes.byref(self.w)

    @property
    def held(self) -> int:
        """Channels an expert holds: cout, or a gated layer's gates and values."""
        return self.cout * (2 if self.w.gated else 1)


def _dtype(t: torch.dtype, name: str) -> int:
    d = DTYPES.get(t)
    if d is None:
        raise ValueError(f"{name}: float32, bfloat16 or float16 expected, got {t}")
    return d


_I32 = 2 ** 31 - 1      # ctypes keeps the low 32 bits of a larger size without a word


def _sizes(name: str, *sizes: int):
    """Raise ValueError where one of them does not fit the library's int32."""
    for v in sizes:
        if not -_I32 - 1 <= v <= _I32:
            raise ValueError(f"{name}: sizes of at most {_I32} expected, got {v}")


def _rows(t: torch.Tensor, name: str, cols: Optional[int] = None):
    """(rows, cols, stride, dtype code) of a 2-d device tensor whose rows are dense."""
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise ValueError(f"{name}: 2-d tensor expected")
    n, c = t.shape
    if n > _I32 or c > _I32:
        _sizes(name, n, c)
    if not t.is_cuda:
        raise ValueError(f"{name}: device tensor expected")
    if cols is not None and c != cols:
        raise ValueError(f"{name}: {cols} columns expected, got {c}")
    stride, inner = t.stride()
    if inner != 1 and c > 1:
        raise ValueError(f"{name}: adjacent elements expected within a row")
    if n <= 1 or stride < c:
        # (one row has no stride, and rows that overlap are for reading only)
        if n > 1:
            raise ValueError(f"{name}: rows that do not overlap expected")
        stride = c
    return n, c, stride, _dtype(t.dtype, name)


def _held(w: torch.Tensor, gated: bool, name: str):
    if w.dim() == 2:
        w = w.unsqueeze(0)
    if w.dim() != 3:
        raise ValueError(f"{name}: [channels, cin] or [experts, channels, cin] expected, got {tuple(w.shape)}")
    e, held, cin = w.shape
    _sizes(name, e, held, cin)
    if gated and held % 2:
        raise ValueError(f"{name}: a gated layer holds its gates and as many values, got {held} channels")
    return w.contiguous(), e, held, cin


def _linear(call: str, e: int, held: int, cin: int, gated: bool, hblock: int, device, run) -> PreparedLinear:
    cout = held // 2 if gated else held
    _sizes("hblock", hblock)
    nbytes = int(load().hatq_linear_weights_bytes(e, cin, cout, int(gated), hblock))
    buf = torch.empty(max(nbytes, 1), dtype=torch.int8, device=device)
    out = LinearWeights()
    _check(run((e, cin, cout, int(gated), hblock), buf.data_ptr(), nbytes, ctypes.byref(out)), call)
    return PreparedLinear(buf, out, e, cin, cout, out.k_stride)


def hatq_prepare_linear(w: torch.Tensor, bias: Optional[torch.Tensor] = None, hblock: int = 1, gated: bool = False,
                        stream=None) -> PreparedLinear:
    """A layer from float weights [held, cin], or experts from [experts, held, cin]
    (bias accordingly).  gated: held = 2 cout, gates first."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hatq_prepare_linear(w, bias, hblock, gated)
    w, e, held, cin = _held(w, gated, "w")
    t = _dtype(w.dtype, "w")
    _need(w, "w", w.dtype, 0)
    b = None if bias is None else bias.contiguous().float()
    _need(b, "bias", torch.float32, e * held, optional=True)
    return _linear("hatq_prepare_linear", e, held, cin, gated, int(hblock), w.device,
                   lambda shape, dst, n, out: load().hatq_prepare_linear(*shape, _ptr(w), t, _ptr(b), dst, n, out,
                                                                         _stream()))


def hatq_pack_linear(codes: torch.Tensor, w_scale: torch.Tensor, bias: Optional[torch.Tensor] = None,
                     hblock: int = 1, gated: bool = False, stream=None) -> PreparedLinear:
    """The same from int8 codes of the transformed weights and their fp32 scales, one
    for each channel (quantized elsewhere)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hatq_pack_linear(codes, w_scale, bias, hblock, gated)
    codes, e, held, cin = _held(codes, gated, "codes")
    _need(codes, "codes", torch.int8, 0)
    s = w_scale.contiguous()
    b = None if bias is None else bias.contiguous()
    _need(s, "w_scale", torch.float32, e * held)
    _need(b, "bias", torch.float32, e * held, optional=True)
    return _linear("hatq_pack_linear", e, held, cin, gated, int(hblock), codes.device,
                   lambda shape, dst, n, out: load().hatq_pack_linear(*shape, _ptr(codes), _ptr(s), _ptr(b), dst, n,
                                                                      out, _stream()))


def hatq_token_quant(x: torch.Tensor, hblock: int = 1, xq: Optional[torch.Tensor] = None,
                     scale: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Tokens x [rows, cin] -> (int8 codes [rows, cin rounded up to 64], a scale for
    each token, fp32 [rows])."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hatq_token_quant(x, hblock, xq, scale)
    n, c, stride, t = _rows(x, "x")
    _sizes("hblock", hblock)
    ks = (c + 63) // 64 * 64
    if xq is None:
        xq = torch.empty((n, ks), dtype=torch.int8, device=x.device)
    if scale is None:
        scale = torch.empty(n, dtype=torch.float32, device=x.device)
    _need(xq, "xq", torch.int8, n * ks)
    _need(scale, "scale", torch.float32, n)
    _check(load().hatq_token_quant(x.data_ptr(), t, n, c, stride, int(hblock), xq.data_ptr(), scale.data_ptr(),
                                   _stream()), "hatq_token_quant")
    return xq, scale


def _out_rows(y: Optional[torch.Tensor], rows: int, cout: int, dtype: torch.dtype, x: torch.Tensor):
    """(y, stride, dtype code) of the output rows, allocated beside x if y is None."""
    if y is None:
        return x.new_empty((rows, cout), dtype=dtype), cout, _dtype(dtype, "out_dtype")
    n, _, stride, t = _rows(y, "y", cout)
    if n != rows:
        raise ValueError(f"y: {rows} rows expected, got {n}")
    return y, stride, t


def _codes(lin: PreparedLinear, xq: torch.Tensor, scale: torch.Tensor) -> int:
    if xq.dim() != 2 or xq.shape[1] != lin.k_stride:
        raise ValueError(f"xq: [rows, {lin.k_stride}] expected, got {tuple(xq.shape)}")
    n = xq.shape[0]
    if n > _I32:
        _sizes("xq", n)
    _need(xq, "xq", torch.int8, 0)
    _need(scale, "scale", torch.float32, n)
    return n


def hatq_linear_int8(lin: PreparedLinear, xq: torch.Tensor, scale: torch.Tensor,
                     out_dtype: torch.dtype = torch.float32, y: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Token codes through one layer: y [rows, cout] of out_dtype (or of the given y)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hatq_linear_int8(lin, xq, scale, out_dtype, y)
    n = _codes(lin, xq, scale)
    y, ys, yt = _out_rows(y, n, lin.cout, out_dtype, xq)
    _check(load().hatq_linear_int8(lin.ref, xq.data_ptr(), scale.data_ptr(), n, y.data_ptr(), yt, ys,
                                   _stream()), "hatq_linear_int8")
    return y


def hatq_linear_ws_bytes(lin: PreparedLinear, rows: int) -> int:
    _sizes("rows", rows)
    return int(load().hatq_linear_ws_bytes(lin.ref, rows))


def _linear_ws(lin, rows: int, ws: Optional[torch.Tensor], x: torch.Tensor) -> torch.Tensor:
    if ws is None:
        # hatq_linear_ws_bytes, without the call
        return x.new_empty(((rows * lin.k_stride + 255) & -256) + ((4 * rows + 255) & -256) or 256, dtype=torch.int8)
    _need(ws, "ws", torch.int8, 0)
    return ws


def hatq_linear_forward(lin: PreparedLinear, x: torch.Tensor, out_dtype: Optional[torch.dtype] = None,
                        y: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Tokens x [rows, cin] through one layer: y [rows, cout] of out_dtype (default: x's)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hatq_linear_forward(lin, x, out_dtype, y, ws)
    n, _, xs, xt = _rows(x, "x", lin.cin)
    y, ys, yt = _out_rows(y, n, lin.cout, out_dtype or x.dtype, x)
    if n <= HATQ_TOKEN_ROWS and n * lin.k_stride <= HATQ_TOKEN_CODES:
        wp, wn = None, 0                # a few tokens need no workspace
    else:
        ws = _linear_ws(lin, n, ws, x)
        wp, wn = ws.data_ptr(), ws.numel()
    _check(load().hatq_linear_forward(lin.ref, x.data_ptr(), xt, n, xs, y.data_ptr(), yt, ys, wp, wn, _stream()),
           "hatq_linear_forward")
    return y


def _grouping(lin: PreparedLinear, ends: torch.Tensor, src: Optional[torch.Tensor], x_rows: int) -> int:
    """The output rows of a grouped call."""
    _need(ends, "ends", torch.int32, lin.experts)
    if src is None:
        return x_rows
    if src.dim() != 1:
        raise ValueError(f"src: 1-d tensor expected, got shape {tuple(src.shape)}")
    _need(src, "src", torch.int32, 0)
    n = src.shape[0]
    if n > _I32:
        _sizes("src", n)
    return n


def hatq_experts_int8(lin: PreparedLinear, xq: torch.Tensor, scale: torch.Tensor, ends: torch.Tensor,
                      src: Optional[torch.Tensor] = None, out_dtype: torch.dtype = torch.float32,
                      y: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Token codes grouped by expert: row i of y is token src[i] (or i) through the first
    expert e with i < ends[e] (int32 [experts], on the device)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hatq_experts_int8(lin, xq, scale, ends, src, out_dtype, y)
    n = _codes(lin, xq, scale)
    rows = _grouping(lin, ends, src, n)
    y, ys, yt = _out_rows(y, rows, lin.cout, out_dtype, xq)
    _check(load().hatq_experts_int8(lin.ref, xq.data_ptr(), scale.data_ptr(), n, ends.data_ptr(), _ptr(src), rows,
                                    y.data_ptr(), yt, ys, _stream()), "hatq_experts_int8")
    return y


def hatq_experts_forward(lin: PreparedLinear, x: torch.Tensor, ends: torch.Tensor,
                         src: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None,
                         y: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """hatq_experts_int8 of the codes of tokens x [x_rows, cin]."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hatq_experts_forward(lin, x, ends, src, out_dtype, y, ws)
    n, _, xs, xt = _rows(x, "x", lin.cin)
    rows = _grouping(lin, ends, src, n)
    y, ys, yt = _out_rows(y, rows, lin.cout, out_dtype or x.dtype, x)
    ws = _linear_ws(lin, n, ws, x)
    _check(load().hatq_experts_forward(lin.ref, x.data_ptr(), xt, n, xs, ends.data_ptr(), _ptr(src), rows,
                                       y.data_ptr(), yt, ys, ws.data_ptr(), ws.numel(), _stream()),
           "hatq_experts_forward")
    return y


def hatq_expert_order(ids: torch.Tensor, experts: int, ends: Optional[torch.Tensor] = None,
                      src: Optional[torch.Tensor] = None, pos: Optional[torch.Tensor] = None,
                      ws: Optional[torch.Tensor] = None, stream=None):
    """Chosen experts ids (int32 [tokens, topk]) -> (ends [experts], src [tokens * topk],
    pos [tokens, topk]): the rows of the grouped calls, sorted by expert.  An id outside
    [0, experts) masks its pair (pos -1)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hatq_expert_order(ids, experts, ends, src, pos, ws)
    if ids.dim() != 2:
        raise ValueError(f"ids: [tokens, topk] expected, got shape {tuple(ids.shape)}")
    _need(ids, "ids", torch.int32, 0)
    t, k = ids.shape
    _sizes("ids, experts", t, k, experts)
    nbytes = int(load().hatq_expert_order_ws_bytes(t, k, experts))
    if ends is None:
        ends = torch.empty(experts, dtype=torch.int32, device=ids.device)
    if src is None:
        src = torch.empty(t * k, dtype=torch.int32, device=ids.device)
    if pos is None:
        pos = torch.empty((t, k), dtype=torch.int32, device=ids.device)
    if ws is None:
        ws = torch.empty(max(nbytes, 1), dtype=torch.int8, device=ids.device)
    _need(ends, "ends", torch.int32, experts)
    _need(src, "src", torch.int32, t * k)
    _need(pos, "pos", torch.int32, t * k)
    _need(ws, "ws", torch.int8, 0)
    _check(load().hatq_expert_order(ids.data_ptr(), t, k, experts, ends.data_ptr(), src.data_ptr(), pos.data_ptr(),
                                    ws.data_ptr(), ws.numel(), _stream()), "hatq_expert_order")
    return ends, src, pos


def hatq_expert_combine(h: torch.Tensor, pos: torch.Tensor, weights: torch.Tensor,
                        out_dtype: torch.dtype = torch.float32, y: Optional[torch.Tensor] = None,
                        stream=None) -> torch.Tensor:
    """y[t] = sum over j of weights[t, j] h[pos[t, j]]: h fp32 [rows, cols], pos int32 and
    weights fp32 [tokens, topk]; a pos outside the rows adds nothing."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hatq_expert_combine(h, pos, weights, out_dtype, y)
    n, c, hs, ht = _rows(h, "h")
    if ht != 0:
        raise ValueError(f"h: float32 expected, got {h.dtype}")
    if pos.dim() != 2 or weights.shape != pos.shape:
        raise ValueError(f"pos, weights: [tokens, topk] expected, got {tuple(pos.shape)}, {tuple(weights.shape)}")
    _need(pos, "pos", torch.int32, 0)
    _need(weights, "weights", torch.float32, 0)
    t, k = pos.shape
    _sizes("pos", t, k)
    y, ys, yt = _out_rows(y, t, c, out_dtype, h)
    _check(load().hatq_expert_combine(h.data_ptr(), n, c, hs, pos.data_ptr(), weights.data_ptr(), t, k, y.data_ptr(),
                                      yt, ys, _stream()), "hatq_expert_combine")
    return y


def hatq_expert_mlp_ws_bytes(w_in: PreparedLinear, w_out: PreparedLinear, tokens: int, topk: int) -> int:
    _sizes("tokens, topk", tokens, topk)
    return int(load().hatq_expert_mlp_ws_bytes(w_in.ref, w_out.ref, tokens, topk))


def hatq_expert_mlp(w_in: PreparedLinear, w_out: PreparedLinear, x: torch.Tensor, ids: torch.Tensor,
                    weights: torch.Tensor, out_dtype: Optional[torch.dtype] = None, y: Optional[torch.Tensor] = None,
                    ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Tokens x [tokens, cin] through their chosen gated experts, ids int32 and weights
    fp32 [tokens, topk]: y [tokens, cout] of out_dtype (default: x's)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hatq_expert_mlp(w_in, w_out, x, ids, weights, out_dtype, y, ws)
    n, _, xs, xt = _rows(x, "x", w_in.cin)
    if ids.dim() != 2 or ids.shape[0] != n or weights.shape != ids.shape:
        raise ValueError(f"ids, weights: [{n}, topk] expected, got {tuple(ids.shape)}, {tuple(weights.shape)}")
    _need(ids, "ids", torch.int32, 0)
    _need(weights, "weights", torch.float32, 0)
    y, ys, yt = _out_rows(y, n, w_out.cout, out_dtype or x.dtype, x)
    topk = ids.shape[1]
    if topk > _I32:
        _sizes("ids", topk)
    if ws is None:
        ws = torch.empty(max(hatq_expert_mlp_ws_bytes(w_in, w_out, n, topk), 256), dtype=torch.int8, device=x.device)
    _need(ws, "ws", torch.int8, 0)
    _check(load().hatq_expert_mlp(w_in.ref, w_out.ref, x.data_ptr(), xt, n, xs, ids.data_ptr(), weights.data_ptr(),
                                  topk, y.data_ptr(), yt, ys, ws.data_ptr(), ws.numel(), _stream()),
           "hatq_expert_mlp")
    return y


_LINEAR4_ROWS = 1 << 24     # the most rows of a call


@dataclass
class PreparedLinear4:
    """Prepared 4-bit linear weights: the device buffer and the C view into it."""
    buf: torch.Tensor
    w: Linear4Weights
    cin: int
    cout: int
    group: int
    k_stride: int

    def __post_init__(self):
        self.ref = ctypes.byref(self.w)
        self.device = self.buf.get_device()
        # the rows up to which a call needs no workspace, as the library has it (of more rows, a call asks
        # hatq_linear4_ws_bytes)
        none, some = 0, 1
        while some <= _LINEAR4_ROWS and not load().hatq_linear4_ws_bytes(self.ref, some):
            none, some = some, 2 * some
        while some - none > 1 and none < _LINEAR4_ROWS:
            half = (none + some) // 2
            none, some = (none, half) if load().hatq_linear4_ws_bytes(self.ref, half) else (half, some)
        self.rows = none


def _linear4(call: str, w: torch.Tensor, gated: bool, hblock: int, group: int, run) -> PreparedLinear4:
    held, cin = w.shape
    cout = held // 2 if gated else held
    _sizes("sizes", held, cin, hblock, group)
    shape = cin, cout, int(gated), hblock, group
    nbytes = int(load().hatq_linear4_weights_bytes(*shape))
    buf = torch.empty(max(nbytes, 1), dtype=torch.int8, device=w.device)
    out = Linear4Weights()
    _check(run(shape, buf.data_ptr(), nbytes, ctypes.byref(out)), call)
    return PreparedLinear4(buf, out, cin, cout, group, out.k_stride)


def _held4(w: torch.Tensor, gated: bool, name: str) -> torch.Tensor:
    if w.dim() != 2:
        raise ValueError(f"{name}: [channels, cin] expected, got {tuple(w.shape)}")
    if gated and w.shape[0] % 2:
        raise ValueError(f"{name}: a gated layer holds its gates and as many values, got {w.shape[0]} channels")
    return w.contiguous()


def hatq_prepare_linear4(w: torch.Tensor, bias: Optional[torch.Tensor] = None, hblock: int = 1, group: int = 128,
                         gated: bool = False, stream=None) -> PreparedLinear4:
    """A layer of 4-bit weights from float weights [held, cin], a scale for each channel and
    `group` input channels (64 or 128).  gated: held = 2 cout, gates first."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hatq_prepare_linear4(w, bias, hblock, group, gated)
    w = _held4(w, gated, "w")
    t = _dtype(w.dtype, "w")
    _need(w, "w", w.dtype, 0)
    b = None if bias is None else bias.contiguous().float()
    _need(b, "bias", torch.float32, w.shape[0], optional=True)
    _here(w.get_device(), b)
    return _linear4("hatq_prepare_linear4", w, gated, hblock, group,
                    lambda shape, dst, n, out: load().hatq_prepare_linear4(*shape, _ptr(w), t, _ptr(b), dst, n, out,
                                                                           _stream()))


def hatq_pack_linear4(codes: torch.Tensor, w_scale: torch.Tensor, bias: Optional[torch.Tensor] = None,
                      hblock: int = 1, gated: bool = False, stream=None) -> PreparedLinear4:
    """The same from int8 codes [held, cin] of the transformed weights, within [-8, 7], and
    their bfloat16 scales [held, groups] (quantized elsewhere); the group is 64 or 128,
    whichever gives as many groups (128 where both do)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hatq_pack_linear4(codes, w_scale, bias, hblock, gated)
    codes = _held4(codes, gated, "codes")
    _need(codes, "codes", torch.int8, 0)
    held, cin = codes.shape
    groups = {-(-cin // g): g for g in (64, 128)}
    if w_scale.dim() != 2 or w_scale.shape[0] != held or w_scale.shape[1] not in groups:
        raise ValueError(f"w_scale: [{held}, {' or '.join(str(g) for g in groups)}] expected, got {tuple(w_scale.shape)}")
    s = w_scale.contiguous()
    b = None if bias is None else bias.contiguous()
    _need(s, "w_scale", torch.bfloat16, 0)
    _need(b, "bias", torch.float32, held, optional=True)
    _here(codes.get_device(), s, b)
    return _linear4("hatq_pack_linear4", codes, gated, hblock, groups[w_scale.shape[1]],
                    lambda shape, dst, n, out: load().hatq_pack_linear4(*shape, _ptr(codes), _ptr(s), _ptr(b), dst, n,
                                                                        out, _stream()))


def hatq_linear4_ws_bytes(lin: PreparedLinear4, rows: int) -> int:
    _sizes("rows", rows)
    return int(load().hatq_linear4_ws_bytes(lin.ref, rows))


def hatq_linear4_forward(lin: PreparedLinear4, x: torch.Tensor, out_dtype: Optional[torch.dtype] = None,
                         y: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                         stream=None) -> torch.Tensor:
    """Tokens x [rows, cin] through a layer of 4-bit weights: y [rows, cout] of out_dtype
    (default: x's)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hatq_linear4_forward(lin, x, out_dtype, y, ws)
    n, _, xs, xt = _rows(x, "x", lin.cin)
    y, ys, yt = _out_rows(y, n, lin.cout, out_dtype or x.dtype, x)
    _here(lin.device, x, y, ws)
    if ws is None and n > lin.rows:
        nbytes = load().hatq_linear4_ws_bytes(lin.ref, n)
        if nbytes:
            ws = x.new_empty(nbytes, dtype=torch.int8)
    _need(ws, "ws", torch.int8, 0, optional=True)
    wp, wn = (None, 0) if ws is None else (ws.data_ptr(), ws.numel())
    _check(load().hatq_linear4_forward(lin.ref, x.data_ptr(), xt, n, xs, y.data_ptr(), yt, ys, wp, wn, _stream()),
           "hatq_linear4_forward")
    return y


@dataclass
class Cache4:
    """A cache of keys and values in 4 bits: the device buffer and the C view of it."""
    buf: torch.Tensor
    c: Cache4View
    pages: int
    page_size: int
    heads: int
    dim: int

    def __post_init__(self):
        self.ref = ctypes.byref(self.c)
        self.device = self.buf.get_device()


def _here(device: int, *tensors: Optional[torch.Tensor]):
    """Raise ValueError unless the tensors are on `device` and it is the current one (the
    calls go to its current stream)."""
    if device != torch._C._cuda_getDevice():
        raise ValueError(f"device {device} expected to be the current one")
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError(f"tensors on device {device} expected, got one on {t.device}")


def hatq_cache4_bytes(pages: int, page_size: int, heads: int, dim: int, hblock: int = 1) -> int:
    _sizes("sizes", pages, page_size, heads, dim, hblock)
    return int(load().hatq_cache4_bytes(pages, page_size, heads, dim, hblock))


def hatq_cache4_init(pages: int, page_size: int, heads: int, dim: int, hblock: int = 1,
                     buf: Optional[torch.Tensor] = None, device="cuda") -> Cache4:
    """A cache of `pages` pages of page_size positions, in the given int8 buffer or a new
    one.  Its contents need no clearing."""
    nbytes = hatq_cache4_bytes(pages, page_size, heads, dim, hblock)
    if buf is None:
        buf = torch.empty(max(nbytes, 1), dtype=torch.int8, device=device)
    _need(buf, "buf", torch.int8, 0)
    out = Cache4View()
    _check(load().hatq_cache4_init(pages, page_size, heads, dim, hblock, buf.data_ptr(), buf.numel(),
                                   ctypes.byref(out)), "hatq_cache4_init")
    return Cache4(buf, out, pages, page_size, heads, dim)


def _heads(t: torch.Tensor, name: str, dim: int, heads: Optional[int] = None, rows: Optional[int] = None):
    """(rows, heads, C view) of a device tensor [rows, heads, dim] with adjacent channels."""
    if not isinstance(t, torch.Tensor) or t.dim() != 3:
        raise ValueError(f"{name}: [rows, heads, {dim}] expected")
    n, h, d = t.shape
    if not t.is_cuda:
        raise ValueError(f"{name}: device tensor expected")
    if d != dim or (heads is not None and h != heads) or (rows is not None and n != rows):
        raise ValueError(f"{name}: [{'rows' if rows is None else rows}, {'heads' if heads is None else heads}, {dim}] "
                         f"expected, got {tuple(t.shape)}")
    if n > _I32 or h > _I32:
        _sizes(name, n, h)
    by_row, by_head, inner = t.stride()
    if inner != 1 and d > 1:
        raise ValueError(f"{name}: adjacent channels expected")
    if h <= 1:
        by_head = d
    if n <= 1:
        by_row = max(h, 1) * by_head
    return n, h, Heads(_dtype(t.dtype, name), by_row, by_head, t.data_ptr())


def _places(cache: Cache4, rows: int, table: torch.Tensor, lens: torch.Tensor, ends: Optional[torch.Tensor]):
    """(batch, width) of the sequences' table."""
    if table.dim() != 2:
        raise ValueError(f"table: [batch, width] expected, got {tuple(table.shape)}")
    batch, width = table.shape
    _need(table, "table", torch.int32, 0)
    _need(lens, "lens", torch.int32, batch)
    _need(ends, "ends", torch.int32, batch, optional=True)
    if batch > _I32 or width > _I32:
        _sizes("table", batch, width)
    if ends is None and batch and rows % batch:
        raise ValueError(f"{rows} rows of {batch} sequences: ends expected")
    return batch, width


def hatq_cache4_append(cache: Cache4, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, lens: torch.Tensor,
                       ends: Optional[torch.Tensor] = None, stream=None) -> None:
    """New tokens' keys and values [rows, heads, dim] into the cache, as the last positions
    of their sequences: table int32 [batch, width], lens int32 [batch] with the new tokens
    counted, ends int32 [batch] the sequences' row ends (None: as many rows each)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hatq_cache4_append(cache, k, v, table, lens, ends)
    n, _, hk = _heads(k, "k", cache.dim, cache.heads)
    _, _, hv = _heads(v, "v", cache.dim, cache.heads, n)
    batch, width = _places(cache, n, table, lens, ends)
    _here(cache.device, k, v, table, lens, ends)
    _check(load().hatq_cache4_append(cache.ref, ctypes.byref(hk), ctypes.byref(hv), n, table.data_ptr(), width,
                                     lens.data_ptr(), _ptr(ends), batch, _stream()), "hatq_cache4_append")


def hatq_cache4_read(cache: Cache4, rows: int, table: torch.Tensor, lens: torch.Tensor,
                     ends: Optional[torch.Tensor] = None, out_dtype: torch.dtype = torch.float32,
                     k: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None,
                     stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """What the cache holds of the sequences' last positions, `rows` of them: keys and values
    [rows, heads, dim] of out_dtype (or of the given k and v).  New tensors are cleared first
    where ends is given, since rows past the last end are not written."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hatq_cache4_read(cache, rows, table, lens, ends, out_dtype, k, v)
    _sizes("rows", rows)
    new = torch.empty if ends is None else torch.zeros
    if k is None and v is None:     # (one allocation, and one launch that clears it)
        k, v = new((2, rows, cache.heads, cache.dim), dtype=out_dtype, device=cache.buf.device).unbind(0)
    elif k is None:
        k = new((rows, cache.heads, cache.dim), dtype=out_dtype, device=cache.buf.device)
    elif v is None:
        v = new((rows, cache.heads, cache.dim), dtype=out_dtype, device=cache.buf.device)
    _, _, hk = _heads(k, "k", cache.dim, cache.heads, rows)
    _, _, hv = _heads(v, "v", cache.dim, cache.heads, rows)
    batch, width = _places(cache, rows, table, lens, ends)
    _here(cache.device, k, v, table, lens, ends)
    _check(load().hatq_cache4_read(cache.ref, ctypes.byref(hk), ctypes.byref(hv), rows, table.data_ptr(), width,
                                   lens.data_ptr(), _ptr(ends), batch, _stream()), "hatq_cache4_read")
    return k, v


def hatq_attention4_ws_bytes(cache: Cache4, rows: int, q_heads: int, width: int, batch: int, ragged: bool = False,
                             window: int = 0, max_len: int = 0) -> int:
    _sizes("sizes", rows, q_heads, width, batch, window, max_len)
    return int(load().hatq_attention4_ws_bytes(cache.ref, rows, q_heads, width, batch, int(ragged), window, max_len))


def hatq_attention4(cache: Cache4, q: torch.Tensor, table: torch.Tensor, lens: torch.Tensor,
                    ends: Optional[torch.Tensor] = None, scale: Optional[float] = None, causal: bool = True,
                    window: int = 0, max_len: int = 0, out_dtype: Optional[torch.dtype] = None,
                    y: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Query rows q [rows, q_heads, dim] over their sequences' positions in the cache: y
    [rows, q_heads, dim] of out_dtype (default: q's).  table, lens, ends as
    hatq_cache4_append, whose tokens the rows are; scale: dim ** -0.5 if None; window: as
    many positions, the row's own the last of them (0: all); max_len: what the lengths will
    not exceed, for the choice of the launch.  A new y is cleared first where ends is given,
    since rows past the last end are not written."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return hatq_attention4(cache, q, table, lens, ends, scale, causal, window, max_len, out_dtype, y, ws)
    n, h, hq = _heads(q, "q", cache.dim)
    if y is None:
        y = (q.new_empty if ends is None else q.new_zeros)((n, h, cache.dim), dtype=out_dtype or q.dtype)
        hy = Heads(_dtype(y.dtype, "y"), max(h, 1) * cache.dim, cache.dim, y.data_ptr())
    else:
        _, _, hy = _heads(y, "y", cache.dim, h, n)
    batch, width = _places(cache, n, table, lens, ends)
    _sizes("window, max_len", window, max_len)
    _here(cache.device, q, y, table, lens, ends, ws)
    if ws is None:
        nbytes = load().hatq_attention4_ws_bytes(cache.ref, n, h, width, batch, int(ends is not None), window, max_len)
        if nbytes:
            ws = torch.empty(nbytes, dtype=torch.int8, device=q.device)
    _need(ws, "ws", torch.int8, 0, optional=True)
    _check(load().hatq_attention4(cache.ref, ctypes.byref(hq), ctypes.byref(hy), n, h, table.data_ptr(), width,
                                  lens.data_ptr(), _ptr(ends), batch, cache.dim ** -0.5 if scale is None else scale,
                                  int(causal), window, max_len, _ptr(ws), 0 if ws is None else ws.numel(), _stream()),
           "hatq_attention4")
    return y
