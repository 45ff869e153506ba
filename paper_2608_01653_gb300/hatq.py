"""Thin Python binding of libhatq (include/hatq.h): argument marshalling only.

Every computation runs inside libhatq's CUDA kernels (or, for the offline
weight preparation, its host code). PyTorch supplies device memory and the
current stream. There is no CPU fallback: if the library cannot be built or
loaded, or no CUDA device is present, the calls raise.
"""
from __future__ import annotations

import ctypes
import re
from dataclasses import dataclass

import numpy as np

from . import build as _build

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_OVERFLOW, ERR_CUDA, ERR_TIMEOUT = range(6)
DH, WH, TRANSFORM = 0, 1, 2
ACT_NONE, ACT_RELU, ACT_SILU, ACT_GELU = 0, 1, 2, 3
IN_OPERAND, IN_I8, IN_F16 = 0, 1, 2

_ACTS = {"none": ACT_NONE, "relu": ACT_RELU, "silu": ACT_SILU, "gelu": ACT_GELU}
GENERAL_ACTS = ("silu", "gelu")
_FORMS = {"DH": DH, "WH": WH}


class HatqError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"hatq status {status}: {message}")
        self.status = status


class ConvDesc(ctypes.Structure):
    _fields_ = [("c_in", ctypes.c_int), ("c_out", ctypes.c_int), ("kh", ctypes.c_int), ("kw", ctypes.c_int),
                ("stride", ctypes.c_int), ("pad", ctypes.c_int), ("form", ctypes.c_int),
                ("hb_in", ctypes.c_int), ("hb_out", ctypes.c_int)]


class PreparedStruct(ctypes.Structure):
    _fields_ = [("d", ConvDesc), ("act", ctypes.c_int), ("hb_next", ctypes.c_int), ("out_f32", ctypes.c_int),
                ("shift", ctypes.c_int), ("k_pad", ctypes.c_int), ("gather", ctypes.c_int),
                ("s_x", ctypes.c_float), ("s_y", ctypes.c_float),
                ("w_i8", ctypes.c_void_p), ("w_f16", ctypes.c_void_p), ("b_int", ctypes.c_void_p),
                ("mult", ctypes.c_void_p), ("deq", ctypes.c_void_p), ("s_w", ctypes.c_void_p),
                ("opaque", ctypes.c_uint64 * 16),
                ("s_z", ctypes.c_float), ("s_u", ctypes.c_float), ("shift_in", ctypes.c_int),
                ("in_affine", ctypes.c_int), ("mult_in", ctypes.c_longlong), ("lut", ctypes.c_int8 * 256),
                ("in_f16", ctypes.c_int), ("out_f16", ctypes.c_int)]


MAX_TRANSPOSED_CLASSES = 4


class PreparedTransposedStruct(ctypes.Structure):
    _fields_ = [("d", ConvDesc), ("out_pad", ctypes.c_int), ("classes", ctypes.c_int),
                ("pad_y", ctypes.c_int * MAX_TRANSPOSED_CLASSES), ("pad_x", ctypes.c_int * MAX_TRANSPOSED_CLASSES),
                ("sub", PreparedStruct * MAX_TRANSPOSED_CLASSES)]


class PreparedGdnStruct(ctypes.Structure):
    _fields_ = [("c", ctypes.c_int), ("inverse", ctypes.c_int), ("hb_next", ctypes.c_int), ("e", ctypes.c_int),
                ("t", ctypes.c_int), ("shift_in", ctypes.c_int), ("P", ctypes.c_longlong),
                ("mult_in", ctypes.c_longlong), ("s_z", ctypes.c_float), ("s_u", ctypes.c_float),
                ("s_y", ctypes.c_float), ("g_f16", ctypes.c_void_p), ("b_pool", ctypes.c_void_p),
                ("opaque", ctypes.c_uint64 * 16)]


class LinearWeightsStruct(ctypes.Structure):
    _fields_ = [("experts", ctypes.c_int), ("n", ctypes.c_int), ("k", ctypes.c_int), ("reserved", ctypes.c_int),
                ("codes", ctypes.c_void_p), ("windows", ctypes.c_void_p), ("s_w", ctypes.c_void_p),
                ("bias", ctypes.c_void_p)]


class TokenCacheStruct(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("pages", ctypes.c_int), ("page", ctypes.c_int), ("heads", ctypes.c_int),
                ("width", ctypes.c_int), ("hb", ctypes.c_int), ("reserved", ctypes.c_int)]


class Linear4WeightsStruct(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int), ("k", ctypes.c_int), ("group", ctypes.c_int), ("reserved", ctypes.c_int),
                ("data", ctypes.c_void_p), ("bias", ctypes.c_void_p)]


_LIB = None
_P = ctypes.c_void_p
_I = ctypes.c_int
_L = ctypes.c_longlong
_F = ctypes.c_float


def load(build: bool = True) -> ctypes.CDLL:
    """Load libhatq.so (building it in-tree first if it is missing or stale)."""
    global _LIB
    if _LIB is None:
        path = _build.build() if build else _build.LIB
        lib = ctypes.CDLL(path)
        sig = {
            "hatq_prepared_sizes": (_I, [ctypes.POINTER(ConvDesc), ctypes.POINTER(ctypes.c_size_t),
                                         ctypes.POINTER(ctypes.c_size_t)]),
            "hatq_prepare_weights": (_I, [ctypes.POINTER(ConvDesc), _P, _P, _F, _F, _I, _I, _I,
                                          ctypes.POINTER(PreparedStruct), _P]),
            "hatq_prepare_weights_general": (_I, [ctypes.POINTER(ConvDesc), _P, _P, _F, _F, _F, _F, _I, _I,
                                                  ctypes.POINTER(PreparedStruct), _P]),
            "hatq_prepare_weights_general_host": (_I, [ctypes.POINTER(ConvDesc), _P, _P, _F, _F, _F, _F, _I, _I,
                                                       _P, _P, _P, _P, _P, ctypes.POINTER(_I),
                                                       ctypes.POINTER(ctypes.c_longlong), ctypes.POINTER(_I), _P]),
            "hatq_prepare_weights_host": (_I, [ctypes.POINTER(ConvDesc), _P, _P, _F, _F, _I, _I, _I,
                                               _P, _P, _P, _P, _P, _P, ctypes.POINTER(_I)]),
            "hatq_quantize_act": (_I, [_P, _I, _F, _I, _I, _I, _I, _I, _F, _P, _P, _P, _P]),
            "hatq_conv2d_i8": (_I, [_P, _I, _I, _I, ctypes.POINTER(PreparedStruct), _P, _P]),
            "hatq_layer": (_I, [_P, _I, _F, _I, _I, _I, ctypes.POINTER(PreparedStruct), _P, _P,
                                ctypes.c_size_t, _P]),
            "hatq_layer_launches": (_I, [_I, _F, ctypes.POINTER(PreparedStruct)]),
            "hatq_last_error": (ctypes.c_char_p, []),
            "hatq_sync_status": (_I, [_P]),
            "hatq_selftest_wait": (_I, [ctypes.c_ulonglong, _P]),
            "hatq_profile_range": (_I, [_P, _I, _I, _I, _I, _I, _P, _P, _P]),
            "hatq_select_form": (_I, [_P, _I, _I, _I, ctypes.POINTER(_I), ctypes.POINTER(_I)]),
            "hatq_hadamard_order": (_I, [_I, ctypes.POINTER(_I)]),
            "hatq_hadamard_matrix": (_I, [_I, _P]),
            "hatq_prepare_weights_order": (_I, [ctypes.POINTER(ConvDesc), _P, _P, _F, _F, _I, _I, _I,
                                                ctypes.POINTER(PreparedStruct), _P]),
            "hatq_prepare_weights_order_host": (_I, [ctypes.POINTER(ConvDesc), _P, _P, _F, _F, _I, _I, _I,
                                                     _P, _P, _P, _P, _P, _P, ctypes.POINTER(_I)]),
            "hatq_prepare_order_transform": (_I, [_I, _F, _F, ctypes.POINTER(PreparedStruct), _P]),
            "hatq_prepare_weights_affine": (_I, [ctypes.POINTER(ConvDesc), _P, _P, _I, ctypes.POINTER(PreparedStruct),
                                                 _P]),
            "hatq_quantize_act_affine": (_I, [_P, _I, _I, _I, _I, _I, _P, _P, _P, _P]),
            "hatq_conv2d_affine": (_I, [_P, _I, _I, _I, ctypes.POINTER(PreparedStruct), _P, _P, _P]),
            "hatq_transposed_sizes": (_I, [ctypes.POINTER(ConvDesc), _I, ctypes.POINTER(ctypes.c_size_t),
                                           ctypes.POINTER(ctypes.c_size_t)]),
            "hatq_prepare_weights_transposed": (_I, [ctypes.POINTER(ConvDesc), _I, _P, _P, _F, _F, _I, _I, _I,
                                                     ctypes.POINTER(PreparedTransposedStruct), _P]),
            "hatq_conv_transpose2d_i8": (_I, [_P, _I, _I, _I, ctypes.POINTER(PreparedTransposedStruct), _P, _P]),
            "hatq_conv2d_i8_subpixel": (_I, [_P, _I, _I, _I, ctypes.POINTER(PreparedStruct), _I, _P, _P]),
            "hatq_layer_noalloc": (_I, [_P, _I, _F, _I, _I, _I, ctypes.POINTER(PreparedStruct), _P, _P]),
            "hatq_prepare_gdn_host": (_I, [_I, _P, _P, _F, _F, _I, _F, _I, _P, _P, ctypes.POINTER(_I),
                                           ctypes.POINTER(ctypes.c_longlong), ctypes.POINTER(_I),
                                           ctypes.POINTER(ctypes.c_longlong), ctypes.POINTER(_I)]),
            "hatq_prepare_gdn": (_I, [_I, _P, _P, _F, _F, _I, _F, _I, ctypes.POINTER(PreparedGdnStruct), _P]),
            "hatq_gdn": (_I, [_P, _I, _I, _I, ctypes.POINTER(PreparedGdnStruct), _P, _P]),
            "hatq_set_operand_format": (_I, [ctypes.POINTER(PreparedStruct), _I, _I]),
            "hatq_quantize_tokens": (_I, [_P, _I, _L, _L, _P, _L, _I, _I, _I, _I, _I, _P, _L, _P, _P]),
            "hatq_linear_sizes": (_I, [_I, _I, _I, ctypes.POINTER(ctypes.c_size_t)]),
            "hatq_linear_layout": (_I, [_P, _L, ctypes.POINTER(LinearWeightsStruct), _P]),
            "hatq_linear_workspace": (_I, [_P, _I, _L, _L, ctypes.POINTER(LinearWeightsStruct),
                                           ctypes.POINTER(ctypes.c_size_t)]),
            "hatq_linear_plan": (_I, [_P, _I, _L, _L, ctypes.POINTER(LinearWeightsStruct), _I, ctypes.c_size_t, _P]),
            "hatq_linear": (_I, [_P, _I, _L, _P, _L, ctypes.POINTER(LinearWeightsStruct), _I, _P, _L, _P,
                                 ctypes.c_size_t, _P]),
            "hatq_grouped_linear": (_I, [_P, _I, _L, _P, _L, _P, ctypes.POINTER(LinearWeightsStruct), _I, _P, _L, _P,
                                         ctypes.c_size_t, _P]),
            "hatq_combine_rows": (_I, [_P, _I, _L, _L, _P, _P, _L, _I, _I, _P, _L, _P]),
            "hatq_append_tokens": (_I, [ctypes.POINTER(TokenCacheStruct), _P, _L, _L, _P, _L, _L, _I, _L, _P, _L, _I, _P, _P,
                                        _I, _P, _P, _P]),
            "hatq_attend_workspace": (_I, [ctypes.POINTER(TokenCacheStruct), _I, _I, _L, _I, _I, _I,
                                           ctypes.POINTER(ctypes.c_size_t)]),
            "hatq_attend_tokens": (_I, [_P, _I, _L, _L, _I, _L, ctypes.POINTER(TokenCacheStruct), _P, _L, _I, _P, _P, _I,
                                        _F, _P, _L, _L, _P, ctypes.c_size_t, _P]),
            "hatq_linear4_sizes": (_I, [_I, _I, _I, ctypes.POINTER(ctypes.c_size_t)]),
            "hatq_quantize_groups": (_I, [_P, _I, _L, _I, _I, _I, _I, _P, _L, _P, _L, _P]),
            "hatq_linear4_layout": (_I, [_P, _L, _P, _L, ctypes.POINTER(Linear4WeightsStruct), _P]),
            "hatq_linear4": (_I, [_P, _I, _L, _P, _L, ctypes.POINTER(Linear4WeightsStruct), _I, _P, _L, _P]),
            "hatq_version": (_I, []),
        }
        for name, (res, args) in sig.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _LIB = lib
    return _LIB


def declared_functions(header_path: str | None = None):
    """Names of the functions include/hatq.h declares."""
    import os
    header_path = header_path or os.path.join(_build.INCLUDE, "hatq.h")
    text = open(header_path).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(hatq_[a-z0-9_]+)\s*\(", text)))


def last_error() -> str:
    return load().hatq_last_error().decode()


def _check(status):
    if status != OK:
        raise HatqError(status, last_error())


def _torch():
    import torch
    if not torch.cuda.is_available():
        raise RuntimeError("libhatq needs a CUDA device; none is available")
    return torch


def _stream(stream):
    torch = _torch()
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else None


def make_desc(c_in, c_out, k, stride, pad, form, hb_in=0, hb_out=0, kw=None) -> ConvDesc:
    form = _FORMS.get(form, form)
    return ConvDesc(c_in, c_out, k, k if kw is None else kw, stride, pad, form, hb_in, hb_out)


def desc_from_spec(spec) -> ConvDesc:
    """A ConvDesc from a layer description with c_in, c_out, k, stride, pad, form, hb_in, hb_out."""
    return make_desc(spec.c_in, spec.c_out, spec.k, spec.stride, spec.pad, spec.form, spec.hb_in, spec.hb_out)


def prepared_sizes(desc: ConvDesc):
    w = ctypes.c_size_t()
    c = ctypes.c_size_t()
    _check(load().hatq_prepared_sizes(ctypes.byref(desc), ctypes.byref(w), ctypes.byref(c)))
    return w.value, c.value


@dataclass
class HostPrepared:
    w_i8: np.ndarray
    w_f16: np.ndarray
    b_int: np.ndarray
    mult: np.ndarray
    deq: np.ndarray
    s_w: np.ndarray
    shift: int


def prepare_weights_host(desc: ConvDesc, w_ohwi, bias, s_x, s_y, act="none", hb_next=0, out_f32=False):
    """hatq_prepare_weights_host: the offline preparation into host arrays."""
    w_elems, ch = prepared_sizes(desc)
    w = np.ascontiguousarray(w_ohwi, dtype=np.float32)
    b = None if bias is None else np.ascontiguousarray(bias, dtype=np.float32)
    out = HostPrepared(np.zeros(w_elems, np.int8), np.zeros(w_elems, np.uint16), np.zeros(ch, np.int32),
                       np.zeros(ch, np.int32), np.zeros(ch, np.float32), np.zeros(ch, np.float32), 0)
    shift = ctypes.c_int()
    _check(load().hatq_prepare_weights_host(
        ctypes.byref(desc), w.ctypes.data, None if b is None else b.ctypes.data, float(s_x), float(s_y),
        _ACTS.get(act, act), int(hb_next), int(bool(out_f32)), out.w_i8.ctypes.data, out.w_f16.ctypes.data,
        out.b_int.ctypes.data, out.mult.ctypes.data, out.deq.ctypes.data, out.s_w.ctypes.data, ctypes.byref(shift)))
    out.shift = shift.value
    k_pad = w_elems // desc.c_out
    out.w_i8 = out.w_i8.reshape(desc.c_out, k_pad)
    out.w_f16 = out.w_f16.reshape(desc.c_out, k_pad)
    return out


class PreparedLayer:
    """A prepared layer: device buffers (torch tensors) plus the C struct."""

    def __init__(self, desc: ConvDesc, device="cuda"):
        torch = _torch()
        w_elems, ch = prepared_sizes(desc)
        self.desc = desc
        self.w_i8 = torch.zeros(w_elems, dtype=torch.int8, device=device)
        self.w_f16 = torch.zeros(w_elems, dtype=torch.float16, device=device)
        self.b_int = torch.zeros(ch, dtype=torch.int32, device=device)
        self.mult = torch.zeros(ch, dtype=torch.int32, device=device)
        self.deq = torch.zeros(ch, dtype=torch.float32, device=device)
        self.s_w = torch.zeros(ch, dtype=torch.float32, device=device)
        self.struct = PreparedStruct()
        self.struct.w_i8 = self.w_i8.data_ptr()
        self.struct.w_f16 = self.w_f16.data_ptr()
        self.struct.b_int = self.b_int.data_ptr()
        self.struct.mult = self.mult.data_ptr()
        self.struct.deq = self.deq.data_ptr()
        self.struct.s_w = self.s_w.data_ptr()

    @property
    def c_in(self):
        return self.desc.c_in

    @property
    def c_out(self):
        return self.desc.c_out

    @property
    def out_f32(self):
        return bool(self.struct.out_f32)

    @property
    def s_x(self):
        return float(self.struct.s_x)

    @property
    def in_f16(self):
        return bool(self.struct.in_f16)

    @property
    def out_f16(self):
        return bool(self.struct.out_f16)

    @property
    def out_dtype(self):
        """torch dtype name of the layer's output tensor."""
        return "float32" if self.out_f32 else ("float16" if self.out_f16 else "int8")

    @property
    def s_y(self):
        return float(self.struct.s_y)

    def out_shape(self, n, h, w):
        d = self.desc
        return (n, (h + 2 * d.pad - d.kh) // d.stride + 1, (w + 2 * d.pad - d.kw) // d.stride + 1, d.c_out)


def prepare_weights(desc: ConvDesc, w_ohwi, bias, s_x, s_y, act="none", hb_next=0, out_f32=False,
                    stream=None, device="cuda", s_z=None, s_u=None) -> PreparedLayer:
    """hatq_prepare_weights (or, for act 'silu' / 'gelu', hatq_prepare_weights_general
    with preactivation scale s_z and activation scale s_u): offline transform,
    quantize and pack into device buffers."""
    L = PreparedLayer(desc, device)
    w = np.ascontiguousarray(w_ohwi, dtype=np.float32)
    b = None if bias is None else np.ascontiguousarray(bias, dtype=np.float32)
    bp = None if b is None else b.ctypes.data
    if act in GENERAL_ACTS:
        if out_f32 or s_z is None or s_u is None:
            raise ValueError("a SiLU / GELU layer emits INT8 codes and needs s_z and s_u")
        _check(load().hatq_prepare_weights_general(ctypes.byref(desc), w.ctypes.data, bp, float(s_x), float(s_z),
                                                   float(s_u), float(s_y), _ACTS[act], int(hb_next),
                                                   ctypes.byref(L.struct), _stream(stream)))
        return L
    _check(load().hatq_prepare_weights(ctypes.byref(desc), w.ctypes.data, bp, float(s_x), float(s_y),
                                       _ACTS.get(act, act), int(hb_next), int(bool(out_f32)),
                                       ctypes.byref(L.struct), _stream(stream)))
    return L


def hadamard_order(c: int) -> int:
    """hatq_hadamard_order: m(C) of Eq. supp_hadamard_order."""
    m = ctypes.c_int()
    _check(load().hatq_hadamard_order(int(c), ctypes.byref(m)))
    return m.value


def hadamard_matrix(m: int) -> np.ndarray:
    """hatq_hadamard_matrix: the library's unnormalized H~_m as an int8 [m, m] array."""
    h = np.zeros((m, m), np.int8)
    _check(load().hatq_hadamard_matrix(int(m), h.ctypes.data))
    return h


def order_desc(desc: ConvDesc) -> ConvDesc:
    """The operand descriptor of a DH layer in the paper's order: c_in = hb_in = m(c_in)."""
    m = hadamard_order(desc.c_in)
    return ConvDesc(m, desc.c_out, desc.kh, desc.kw, desc.stride, desc.pad, desc.form, m, 0)


def prepare_weights_order_host(desc: ConvDesc, w_ohwi, bias, s_x, s_y, act="none", hb_next=0, out_f32=False):
    """hatq_prepare_weights_order_host: a paper-order DH layer prepared into host arrays."""
    if desc.form != DH:                             # the library rejects it before touching any buffer
        _check(load().hatq_prepare_weights_order_host(ctypes.byref(desc), None, None, float(s_x), float(s_y), 0, 0,
                                                      0, None, None, None, None, None, None, None))
    dop = order_desc(desc)
    w_elems, ch = prepared_sizes(dop)
    w = np.ascontiguousarray(w_ohwi, dtype=np.float32)
    b = None if bias is None else np.ascontiguousarray(bias, dtype=np.float32)
    out = HostPrepared(np.zeros(w_elems, np.int8), np.zeros(w_elems, np.uint16), np.zeros(ch, np.int32),
                       np.zeros(ch, np.int32), np.zeros(ch, np.float32), np.zeros(ch, np.float32), 0)
    shift = ctypes.c_int()
    _check(load().hatq_prepare_weights_order_host(
        ctypes.byref(desc), w.ctypes.data, None if b is None else b.ctypes.data, float(s_x), float(s_y),
        _ACTS.get(act, act), int(hb_next), int(bool(out_f32)), out.w_i8.ctypes.data, out.w_f16.ctypes.data,
        out.b_int.ctypes.data, out.mult.ctypes.data, out.deq.ctypes.data, out.s_w.ctypes.data, ctypes.byref(shift)))
    out.shift = shift.value
    out.w_i8 = out.w_i8.reshape(desc.c_out, -1)
    out.w_f16 = out.w_f16.reshape(desc.c_out, -1)
    return out


def prepare_weights_order(desc: ConvDesc, w_ohwi, bias, s_x, s_y, act="none", hb_next=0, out_f32=False,
                          stream=None, device="cuda") -> "PreparedLayer":
    """hatq_prepare_weights_order: a DH layer whose input side takes the paper's
    order m(c_in); the returned layer consumes an operand of m channels."""
    L = PreparedLayer(order_desc(desc), device)
    w = np.ascontiguousarray(w_ohwi, dtype=np.float32)
    b = None if bias is None else np.ascontiguousarray(bias, dtype=np.float32)
    _check(load().hatq_prepare_weights_order(ctypes.byref(desc), w.ctypes.data, None if b is None else b.ctypes.data,
                                             float(s_x), float(s_y), _ACTS.get(act, act), int(hb_next),
                                             int(bool(out_f32)), ctypes.byref(L.struct), _stream(stream)))
    return L


def prepare_order_transform(c: int, s_in, s_out, stream=None, device="cuda") -> "PreparedLayer":
    """hatq_prepare_order_transform: the activation-side transform into the
    order m(c) as a 1x1 layer (c -> m channels), run with conv2d_i8 or layer."""
    m = hadamard_order(c)
    L = PreparedLayer(ConvDesc(c, m, 1, 1, 1, 0, TRANSFORM, 0, 0), device)
    _check(load().hatq_prepare_order_transform(int(c), float(s_in), float(s_out), ctypes.byref(L.struct),
                                               _stream(stream)))
    return L


def prepare_weights_affine(desc: ConvDesc, w_ohwi, bias, act="none", stream=None, device="cuda") -> "PreparedLayer":
    """hatq_prepare_weights_affine: a layer for dynamic affine activations
    (centred int16 operand, per-input scale, float32 output)."""
    L = PreparedLayer(desc, device)
    w = np.ascontiguousarray(w_ohwi, dtype=np.float32)
    b = None if bias is None else np.ascontiguousarray(bias, dtype=np.float32)
    _check(load().hatq_prepare_weights_affine(ctypes.byref(desc), w.ctypes.data, None if b is None else b.ctypes.data,
                                              _ACTS.get(act, act), ctypes.byref(L.struct), _stream(stream)))
    return L


def quantize_act_affine(x, hb, y=None, params=None, workspace=None, stream=None):
    """hatq_quantize_act_affine on a CUDA fp16 NHWC tensor: returns (centred
    int16 codes, params = device float[2] holding s and z)."""
    if getattr(x, "dim", lambda: 0)() != 4:
        raise ValueError("x must be a 4-D NHWC tensor")
    _check_tensor(x, "x", "float16")
    n, h, w, c = x.shape
    if y is not None:
        _check_tensor(y, "y", "int16", (n, h, w, c))
    _check_cuda(("x", x), ("y", y))
    torch = _torch()
    if y is None:
        y = torch.empty((n, h, w, c), dtype=torch.int16, device=x.device)
    if params is None:
        params = torch.empty(2, dtype=torch.float32, device=x.device)
    if workspace is None:
        workspace = torch.empty(64, dtype=torch.uint8, device=x.device)
    _check(load().hatq_quantize_act_affine(_ptr(x), n, h, w, c, int(hb), _ptr(y), _ptr(params), _ptr(workspace),
                                           _stream(stream)))
    return y, params


def conv2d_affine(x, L: "PreparedLayer", params, y=None, stream=None):
    """hatq_conv2d_affine: the convolution on centred int16 codes at step params[0]."""
    if getattr(x, "dim", lambda: 0)() != 4 or x.shape[-1] != L.c_in:
        raise ValueError("x must be a 4-D NHWC tensor with the layer's input channels")
    _check_tensor(x, "x", "int16")
    n, h, w, c = x.shape
    if y is not None:
        _check_tensor(y, "y", "float32", L.out_shape(n, h, w))
    _check_cuda(("x", x), ("y", y), ("params", params))
    torch = _torch()
    if y is None:
        y = torch.empty(L.out_shape(n, h, w), dtype=torch.float32, device=x.device)
    _check(load().hatq_conv2d_affine(_ptr(x), n, h, w, ctypes.byref(L.struct), _ptr(params), _ptr(y), _stream(stream)))
    return y


class PreparedTransposed:
    """A prepared transposed convolution: one sub-layer (device buffers + C
    struct) per output parity class, inside the C struct
    hatq_prepared_transposed."""

    def __init__(self, desc: ConvDesc, out_pad: int, device="cuda"):
        torch = _torch()
        self.desc = desc
        self.out_pad = out_pad
        self.struct = PreparedTransposedStruct()
        self.buffers = []
        for cls in range(desc.stride * desc.stride):
            w = ctypes.c_size_t()
            c = ctypes.c_size_t()
            _check(load().hatq_transposed_sizes(ctypes.byref(desc), cls, ctypes.byref(w), ctypes.byref(c)))
            bufs = dict(w_i8=torch.zeros(w.value, dtype=torch.int8, device=device),
                        w_f16=torch.zeros(w.value, dtype=torch.float16, device=device),
                        b_int=torch.zeros(c.value, dtype=torch.int32, device=device),
                        mult=torch.zeros(c.value, dtype=torch.int32, device=device),
                        deq=torch.zeros(c.value, dtype=torch.float32, device=device),
                        s_w=torch.zeros(c.value, dtype=torch.float32, device=device))
            for k, t in bufs.items():
                setattr(self.struct.sub[cls], k, t.data_ptr())
            self.buffers.append(bufs)

    @property
    def c_in(self):
        return self.desc.c_in

    @property
    def out_f32(self):
        return bool(self.struct.sub[0].out_f32)

    def out_shape(self, n, h, w):
        d = self.desc
        return (n, (h - 1) * d.stride - 2 * d.pad + d.kh + self.out_pad,
                (w - 1) * d.stride - 2 * d.pad + d.kw + self.out_pad, d.c_out)


def prepare_weights_transposed(desc: ConvDesc, out_pad, w_ohwi, bias, s_x, s_y, act="none", hb_next=0,
                               out_f32=False, stream=None, device="cuda") -> PreparedTransposed:
    """hatq_prepare_weights_transposed: a transposed convolution (decoder side)
    prepared as one stride-1 sub-layer per output parity class."""
    T = PreparedTransposed(desc, out_pad, device)
    w = np.ascontiguousarray(w_ohwi, dtype=np.float32)
    b = None if bias is None else np.ascontiguousarray(bias, dtype=np.float32)
    _check(load().hatq_prepare_weights_transposed(ctypes.byref(desc), int(out_pad), w.ctypes.data,
                                                  None if b is None else b.ctypes.data, float(s_x), float(s_y),
                                                  _ACTS.get(act, act), int(hb_next), int(bool(out_f32)),
                                                  ctypes.byref(T.struct), _stream(stream)))
    return T


def conv_transpose2d_i8(x, T: PreparedTransposed, y=None, stream=None):
    """hatq_conv_transpose2d_i8 on the INT8 operand x (NHWC)."""
    n, h, w, c = _check_layer_io(x, IN_OPERAND, T, y)
    torch = _torch()
    if y is None:
        y = torch.empty(T.out_shape(n, h, w), dtype=torch.float32 if T.out_f32 else torch.int8, device=x.device)
    _check(load().hatq_conv_transpose2d_i8(_ptr(x), n, h, w, ctypes.byref(T.struct), _ptr(y), _stream(stream)))
    return y


@dataclass
class HostGdn:
    """hatq_prepare_gdn_host outputs."""
    G: np.ndarray
    B: np.ndarray
    e: int
    P: int
    t: int
    mult_in: int
    shift_in: int


def _gdn_args(c, beta, gamma):
    beta = np.ascontiguousarray(beta, dtype=np.float64).ravel()
    gamma = np.ascontiguousarray(gamma, dtype=np.float64)
    if beta.size != c or gamma.shape != (c, c):
        raise ValueError(f"beta must have {c} entries and gamma be {c} x {c}")
    return beta, gamma


def prepare_gdn_host(c, beta, gamma, s_z, s_u, inverse, s_y, hb_next=0) -> HostGdn:
    """hatq_prepare_gdn_host: the integer GDN / IGDN parameters on the host."""
    beta, gamma = _gdn_args(c, beta, gamma)
    G = np.zeros((c, c), dtype=np.int32)
    B = np.zeros(c, dtype=np.int32)
    e, t, n_in = _I(), _I(), _I()
    P, m_in = ctypes.c_longlong(), ctypes.c_longlong()
    _check(load().hatq_prepare_gdn_host(int(c), beta.ctypes.data, gamma.ctypes.data, float(s_z), float(s_u),
                                        int(bool(inverse)), float(s_y), int(hb_next), G.ctypes.data, B.ctypes.data,
                                        ctypes.byref(e), ctypes.byref(P), ctypes.byref(t), ctypes.byref(m_in),
                                        ctypes.byref(n_in)))
    return HostGdn(G, B, e.value, P.value, t.value, m_in.value, n_in.value)


class PreparedGdn:
    """A prepared GDN / IGDN transition: device G (fp16) and B, and the C
    struct hatq_prepared_gdn."""

    def __init__(self, c, device="cuda"):
        torch = _torch()
        self.c = c
        self.g_f16 = torch.zeros(c * c, dtype=torch.float16, device=device)
        self.b_pool = torch.zeros(c, dtype=torch.int32, device=device)
        self.struct = PreparedGdnStruct()
        self.struct.g_f16 = self.g_f16.data_ptr()
        self.struct.b_pool = self.b_pool.data_ptr()


def prepare_gdn(c, beta, gamma, s_z, s_u, inverse, s_y, hb_next=0, stream=None, device="cuda") -> PreparedGdn:
    """hatq_prepare_gdn: phi_int of GDN (inverse False) or IGDN for c channels
    and the next layer's input transition (block hb_next, scale s_y)."""
    beta, gamma = _gdn_args(c, beta, gamma)
    g = PreparedGdn(c, device)
    _check(load().hatq_prepare_gdn(int(c), beta.ctypes.data, gamma.ctypes.data, float(s_z), float(s_u),
                                   int(bool(inverse)), float(s_y), int(hb_next), ctypes.byref(g.struct),
                                   _stream(stream)))
    return g


def gdn(z, g: PreparedGdn, y=None, stream=None):
    """hatq_gdn on the preactivation codes z (NHWC int8, c channels): the
    next layer's INT8 operand."""
    _check_tensor(z, "z", "int8")
    if z.dim() != 4 or z.shape[-1] != g.c:
        raise ValueError(f"z must be NHWC with {g.c} channels")
    if y is not None:
        _check_tensor(y, "y", "int8", tuple(z.shape))
    _check_cuda(("z", z), ("y", y))
    torch = _torch()
    if y is None:
        y = torch.empty_like(z)
    n, h, w, _ = z.shape
    _check(load().hatq_gdn(_ptr(z), n, h, w, ctypes.byref(g.struct), _ptr(y), _stream(stream)))
    return y


def conv2d_i8_subpixel(x, L: "PreparedLayer", r: int, y=None, stream=None):
    """hatq_conv2d_i8_subpixel: the convolution followed by the sub-pixel
    (depth-to-space) rearrangement with factor r, in the copy-out."""
    n, h, w, c = _check_layer_io(x, IN_OPERAND, L, None)
    _, ho, wo, co = L.out_shape(n, h, w)
    shape = (n, ho * r, wo * r, co // (r * r))
    if y is not None:
        _check_tensor(y, "y", "int8", shape)
    torch = _torch()
    if y is None:
        y = torch.empty(shape, dtype=torch.int8, device=x.device)
    _check(load().hatq_conv2d_i8_subpixel(_ptr(x), n, h, w, ctypes.byref(L.struct), int(r), _ptr(y), _stream(stream)))
    return y


@dataclass
class HostGeneral:
    w_i8: np.ndarray
    b_int: np.ndarray
    mult: np.ndarray
    s_w: np.ndarray
    shift: int
    mult_in: int
    shift_in: int
    lut: np.ndarray


def prepare_weights_general_host(desc: ConvDesc, w_ohwi, bias, s_x, s_z, s_u, s_y, act, hb_next=0) -> HostGeneral:
    """hatq_prepare_weights_general_host: the host half of a SiLU / GELU layer's preparation."""
    w_elems, ch = prepared_sizes(desc)
    w = np.ascontiguousarray(w_ohwi, dtype=np.float32)
    b = None if bias is None else np.ascontiguousarray(bias, dtype=np.float32)
    w_i8, w_f16 = np.zeros(w_elems, np.int8), np.zeros(w_elems, np.uint16)
    b_int, mult, s_w = np.zeros(ch, np.int32), np.zeros(ch, np.int32), np.zeros(ch, np.float32)
    lut = np.zeros(256, np.int8)
    shift, shift_in, mult_in = ctypes.c_int(), ctypes.c_int(), ctypes.c_longlong()
    _check(load().hatq_prepare_weights_general_host(
        ctypes.byref(desc), w.ctypes.data, None if b is None else b.ctypes.data, float(s_x), float(s_z), float(s_u),
        float(s_y), _ACTS[act], int(hb_next), w_i8.ctypes.data, w_f16.ctypes.data, b_int.ctypes.data,
        mult.ctypes.data, s_w.ctypes.data, ctypes.byref(shift), ctypes.byref(mult_in), ctypes.byref(shift_in),
        lut.ctypes.data))
    return HostGeneral(w_i8.reshape(desc.c_out, -1), b_int, mult, s_w, shift.value, mult_in.value, shift_in.value, lut)


_KIND_DTYPE = {IN_OPERAND: "int8", IN_I8: "int8", IN_F16: "float16"}


def _check_tensor(t, what, dtype=None, shape=None):
    """Shape, dtype, layout and device of a tensor handed to the library: the
    entry points read and write exactly the elements these describe."""
    import torch
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{what} must be a torch tensor")
    if dtype is not None and t.dtype != getattr(torch, dtype):
        raise ValueError(f"{what} must be {dtype}, got {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous (NHWC, C innermost)")


def _check_cuda(*named):
    for what, t in named:
        if t is not None and not t.is_cuda:
            raise ValueError(f"{what} must be on a CUDA device")


def _check_layer_io(x, x_kind, L, y=None, scratch=None):
    """The input of a layer call (kind, dtype, 4-D NHWC with L.c_in channels)
    and, when given, its output and scratch buffers."""
    if x_kind not in _KIND_DTYPE:
        raise ValueError(f"unknown input kind {x_kind}")
    if getattr(x, "dim", lambda: 0)() != 4:
        raise ValueError("x must be a 4-D NHWC tensor")
    n, h, w, c = x.shape
    if c != L.c_in:
        raise ValueError(f"x has {c} channels, the layer takes {L.c_in}")
    f16_op = x_kind == IN_OPERAND and getattr(L, "in_f16", False)
    _check_tensor(x, "x", "float16" if f16_op else _KIND_DTYPE[x_kind])
    if y is not None:
        _check_tensor(y, "y", getattr(L, "out_dtype", "float32" if L.out_f32 else "int8"), L.out_shape(n, h, w))
    if scratch is not None:
        _check_tensor(scratch, "scratch", "int8")
    _check_cuda(("x", x), ("y", y), ("scratch", scratch))
    return n, h, w, c


def quantize_act(x, x_kind, s_in, hb, s_out, y=None, s_used=None, workspace=None, stream=None):
    """hatq_quantize_act on a CUDA NHWC tensor (int8 codes or fp16 values).
    s_out <= 0 selects the dynamic mode (s_used: 1-element float32 CUDA tensor)."""
    torch = _torch()
    if x_kind not in (IN_I8, IN_F16) or getattr(x, "dim", lambda: 0)() != 4:
        raise ValueError("x must be a 4-D NHWC tensor of kind IN_I8 or IN_F16")
    _check_tensor(x, "x", _KIND_DTYPE[x_kind])
    n, h, w, c = x.shape
    if y is not None:
        _check_tensor(y, "y", "int8", (n, h, w, c))
    _check_cuda(("x", x), ("y", y))
    if y is None:
        y = torch.empty((n, h, w, c), dtype=torch.int8, device=x.device)
    if s_out <= 0:
        if s_used is None:
            s_used = torch.empty(1, dtype=torch.float32, device=x.device)
        if workspace is None:
            workspace = torch.empty(64, dtype=torch.uint8, device=x.device)
    _check(load().hatq_quantize_act(_ptr(x), int(x_kind), float(s_in), n, h, w, c, int(hb), float(s_out), _ptr(y),
                                    _ptr(s_used), _ptr(workspace), _stream(stream)))
    return (y, s_used) if s_out <= 0 else y


def set_operand_format(L: PreparedLayer, in_f16: bool, out_f16: bool):
    """hatq_set_operand_format: the layer's operand (in_f16) and / or its
    output codes (out_f16) stored as fp16 values instead of int8."""
    _check(load().hatq_set_operand_format(ctypes.byref(L.struct), int(bool(in_f16)), int(bool(out_f16))))
    return L


def conv2d_i8(x, L: PreparedLayer, y=None, stream=None):
    """hatq_conv2d_i8: convolution + fused requantize epilogue on the INT8 operand x (NHWC; fp16 codes
    for a layer with in_f16)."""
    n, h, w, c = _check_layer_io(x, IN_OPERAND, L, y)
    torch = _torch()
    if y is None:
        y = torch.empty(L.out_shape(n, h, w), dtype=getattr(torch, L.out_dtype), device=x.device)
    _check(load().hatq_conv2d_i8(_ptr(x), n, h, w, ctypes.byref(L.struct), _ptr(y), _stream(stream)))
    return y


def layer(x, x_kind, s_in, L: PreparedLayer, y=None, scratch=None, stream=None):
    """hatq_layer: input transform/quantize (when needed) + conv in one call."""
    n, h, w, c = _check_layer_io(x, x_kind, L, y, scratch)
    torch = _torch()
    if y is None:
        y = torch.empty(L.out_shape(n, h, w), dtype=getattr(torch, L.out_dtype), device=x.device)
    nbytes = 0
    if layer_launches(x_kind, s_in, L) > 1:
        if scratch is None:
            scratch = torch.empty(n * h * w * c, dtype=torch.int8, device=x.device)
        nbytes = scratch.numel() * scratch.element_size()
    _check(load().hatq_layer(_ptr(x), int(x_kind), float(s_in), n, h, w, ctypes.byref(L.struct), _ptr(y),
                             _ptr(scratch), nbytes, _stream(stream)))
    return y


def layer_launches(x_kind, s_in, L: PreparedLayer) -> int:
    return int(load().hatq_layer_launches(int(x_kind), float(s_in), ctypes.byref(L.struct)))


def sync_status(stream=None):
    _check(load().hatq_sync_status(_stream(stream)))


def profile_range(x, hb: int, stream=None):
    """hatq_profile_range on an NHWC int8 code tensor: returns (maxima [n, 2]
    int32: max|x_k|, max|H~ x_k| per image; expands [n] uint8)."""
    import torch
    if x.dtype != torch.int8 or x.dim() != 4 or not x.is_cuda:
        raise ValueError("x must be a CUDA int8 NHWC tensor")
    x = x.contiguous()
    n, h, w, c = x.shape
    maxima = torch.empty((n, 2), dtype=torch.int32, device=x.device)
    expands = torch.empty((n,), dtype=torch.uint8, device=x.device)
    _check(load().hatq_profile_range(_ptr(x), n, h, w, c, hb, _ptr(maxima), _ptr(expands), _stream(stream)))
    return maxima, expands


def select_form(expands, tau=(4, 5)):
    """hatq_select_form: the DH/WH decision of Eq. layerwise_hadamard_selection
    from the per-image indicators (host array or tensor) and tau_sel given as
    (numerator, denominator). Returns (form 'DH' or 'WH', p_l as a Fraction)."""
    from fractions import Fraction
    e = np.ascontiguousarray(expands.cpu().numpy() if hasattr(expands, "cpu") else expands, dtype=np.uint8).ravel()
    form, count = ctypes.c_int(), ctypes.c_int()
    _check(load().hatq_select_form(e.ctypes.data if e.size else None, int(e.size), int(tau[0]), int(tau[1]),
                                   ctypes.byref(form), ctypes.byref(count)))
    return ("WH" if form.value == WH else "DH"), Fraction(count.value, int(e.size))


def selftest_wait(limit_cycles: int, stream=None):
    """hatq_selftest_wait: make one bounded device wait expire on purpose
    (failure-detection test; the next sync_status() raises ERR_TIMEOUT)."""
    _check(load().hatq_selftest_wait(int(limit_cycles), _stream(stream)))


def version() -> int:
    return int(load().hatq_version())


def layer_noalloc(x, x_kind, s_in, L: PreparedLayer, y=None, stream=None):
    """hatq_layer_noalloc: hatq_layer for callers that cannot allocate device
    memory; the staged INT8 operand lives in the library's fixed device array
    (at most HATQ_NOALLOC_MAX_BYTES bytes, shared by all calls)."""
    n, h, w, c = _check_layer_io(x, x_kind, L, y)
    torch = _torch()
    if y is None:
        y = torch.empty(L.out_shape(n, h, w), dtype=getattr(torch, L.out_dtype), device=x.device)
    _check(load().hatq_layer_noalloc(_ptr(x), int(x_kind), float(s_in), n, h, w, ctypes.byref(L.struct), _ptr(y),
                                     _stream(stream)))
    return y


NOALLOC_MAX_BYTES = 32 << 20


# ------------------------------------------------------------------ token layers

F32, F16, BF16 = 0, 1, 2
CODES_I8, CODES_F16 = 0, 1

_CODE_FORMATS = {"i8": CODES_I8, "f16": CODES_F16}
_TOKEN_TYPES = {}                                   # torch dtype -> hatq_type / hatq_codes, filled on first use
_CODE_TYPES = {}
_TORCH = None


# A decode step's kernels run for a few microseconds, so the checks of a call are kept to what takes tens of
# nanoseconds each: no tensor is made, no device object compared, no symbol imported.

def _token_torch():
    """torch, with the dtype tables filled (this module imports without torch)."""
    global _TORCH
    if _TORCH is None:
        import torch
        _CODE_TYPES.update({torch.int8: CODES_I8, torch.float16: CODES_F16})
        _TOKEN_TYPES.update({torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16})
        _TORCH = torch
    return _TORCH


def _rows_of(t, name, types, device):
    """Checks a [rows][values] tensor on `device` with contiguous rows; returns its type code, its rows, the values of
    a row and the pitch in elements (below the values where rows overlap or are one row, as expand makes them)."""
    code = types.get(t.dtype)
    if code is None:
        raise ValueError(f"{name}: dtype {t.dtype} is none of {[str(d) for d in types]}")
    if t.dim() != 2:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected two dimensions")
    if t.get_device() != device:
        raise ValueError(f"{name}: on {t.device}, expected cuda:{device}")
    rows, values = t.shape
    pitch, inner = t.stride()
    if inner != 1 and values > 1:
        raise ValueError(f"{name}: the values of a row must be contiguous")
    return code, rows, values, pitch if rows > 1 else values     # a single row may carry any stride


def _out_of(t, types, rows, values, device):
    """Checks a tensor to write [rows][values] into; returns its type code and its pitch."""
    code, r, v, pitch = _rows_of(t, "out", types, device)
    if r != rows or v != values:
        raise ValueError(f"out: shape {(r, v)}, expected {(rows, values)}")
    if pitch < values:
        raise ValueError(f"out: rows overlap (stride {pitch} for {values} values)")
    return code, pitch


def _apart(t, stream):
    """A copy whose rows lie apart, as the library takes them, made on the stream that the call runs on."""
    if stream is None:
        return t.contiguous()
    with _TORCH.cuda.stream(stream):
        return t.contiguous()


def _flat(t, name, dtype, shape, device):
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != device:
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor of shape {tuple(shape)} on cuda:{device}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _launch_stream(t, stream):
    """(device index, raw stream) of a call: `stream`, or the device's current one. The device must be the current one."""
    torch = _token_torch()
    device = t.get_device()
    if device < 0:
        raise ValueError(f"expected CUDA tensors, got {t.device}")
    if device != torch._C._cuda_getDevice():
        raise ValueError(f"the tensors are on cuda:{device}, the current device is cuda:{torch.cuda.current_device()}")
    return device, torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream


def _empty(like, shape, dtype, stream):
    """A tensor of a call's own; it belongs to the stream that the call runs on."""
    if stream is None:
        return _TORCH.empty(shape, dtype=dtype, device=like.device)
    with _TORCH.cuda.stream(stream):
        return _TORCH.empty(shape, dtype=dtype, device=like.device)


class LinearWeights:
    """The weights of a token layer (hatq_linear_weights): device buffers and the C struct."""

    def __init__(self, experts, n, k, codes, windows, s_w, bias, grouped):
        self.experts, self.n, self.k, self.grouped = experts, n, k, grouped
        self.codes, self.windows, self.s_w, self.bias = codes, windows, s_w, bias
        self.device = codes.get_device()
        self.size, self.row_bytes = n * k, 2 * (-(-k // 64) * 64)    # products per row; hatq_linear's workspace
        self.struct = LinearWeightsStruct(experts, n, k, 0, codes.data_ptr(), windows.data_ptr(), s_w.data_ptr(),
                                          None if bias is None else bias.data_ptr())
        self.ref = ctypes.byref(self.struct)


def _per_channel(t, name, e, n, device):
    """A float32 copy of one value per output channel: [experts][n] (dense: or [n]), flat, or with a reduced k kept."""
    shape = tuple(t.shape)
    if t.numel() != e * n or not (t.dim() <= 1 or shape[:2] == (e, n) or e == 1 and shape[0] == n):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected one value per output channel, {(e, n)}")
    return t.to(device=device, dtype=_TORCH.float32).reshape(-1).clone()


def prepare_linear(w, hb=1, scales=None, bias=None, stream=None) -> LinearWeights:
    """The weights of linear (w [n][k]) or grouped_linear (w [experts][n][k]), on the device.

    w in float32 / float16 / bfloat16 (k <= 32768) is transformed along k in blocks
    of hb and quantized with one scale per output channel, as hatq_quantize_tokens
    does with a row; quantize_tokens must be called with the same hb. w in int8 is
    taken as it is, with `scales` ([n] or [experts][n], float32). bias: [n] or
    [experts][n], any floating type."""
    torch = _token_torch()
    _torch()
    if w.dim() not in (2, 3):
        raise ValueError(f"w: shape {tuple(w.shape)}, expected [n, k] or [experts, n, k]")
    grouped = w.dim() == 3
    e, n, k = w.shape if grouped else (1, *w.shape)
    size = ctypes.c_size_t()
    _check(load().hatq_linear_sizes(e, n, k, ctypes.byref(size)))
    device, raw = _launch_stream(w, stream)
    with torch.cuda.stream(stream):                 # None: the current one
        rows = w.reshape(e * n, k)
        if k > 1 and rows.stride(1) != 1 or rows.stride(0) < k:
            rows = rows.contiguous()
        if w.dtype == torch.int8:
            if scales is None or hb != 1:
                raise ValueError("int8 weights need their scales, and are not transformed")
            s_w = _per_channel(scales, "scales", e, n, w.device)
        else:
            if scales is not None:
                raise ValueError("scales belong to int8 weights")
            rows, s_w = quantize_tokens(rows, hb=hb, codes="i8", stream=stream)
        b = None if bias is None else _per_channel(bias, "bias", e, n, w.device)
        pitch = rows.stride(0) if e * n > 1 else k
        L = LinearWeights(e, n, k, torch.empty(size.value, dtype=torch.uint8, device=w.device),
                          torch.empty(e, dtype=torch.int32, device=w.device), s_w, b, grouped)
        _check(load().hatq_linear_layout(rows.data_ptr(), pitch, L.ref, raw))
    return L


def quantize_tokens(x, hb=1, act="none", gated=False, rows=None, codes="auto", out=None, scales=None, stream=None):
    """hatq_quantize_tokens: (codes, scales) of the rows of x ([rows][c], or [rows][2 c] when gated).

    rows: int32 [n], the source row of each output row (outside x: an empty row).
    codes: "i8", "f16", or "auto": int8 for up to 2 rows (the dot-product kernel
    reads them as they are), fp16 above (the tensor cores do). out / scales:
    tensors to write into; new codes come with a pitch that suits the products."""
    torch = _TORCH or _token_torch()
    device, raw = _launch_stream(x, stream)
    kind, src_rows, c, pitch = _rows_of(x, "x", _TOKEN_TYPES, device)
    if pitch < c:
        x, pitch = _apart(x, stream), c
    code = _ACTS.get(act)
    if code is None:
        raise ValueError(f"unknown activation {act!r}")
    if gated:
        if c % 2:
            raise ValueError("a gated row holds two halves")
        c //= 2
    if rows is None:
        n, index = src_rows, None
    else:
        n = rows.shape[0]
        index = _flat(rows, "rows", torch.int32, (n,), device)
    if codes == "auto":
        codes = "i8" if n <= 2 else "f16"
    fmt = _CODE_FORMATS.get(codes)
    if fmt is None:
        raise ValueError(f"unknown code format {codes!r}")
    if out is None:
        out_pitch = -(-c // 16) * 16 if fmt == CODES_I8 else -(-c // 8) * 8
        out = _empty(x, (n, out_pitch), torch.int8 if fmt == CODES_I8 else torch.float16, stream)
        if out_pitch != c:
            out = out[:, :c]
    else:
        kept, out_pitch = _out_of(out, _CODE_TYPES, n, c, device)
        if kept != fmt:
            raise ValueError(f"out: {out.dtype} does not hold {codes} codes")
    if scales is None:
        scales = _empty(x, (n,), torch.float32, stream)
        ps = scales.data_ptr()
    else:
        ps = _flat(scales, "scales", torch.float32, (n,), device)
    st = (_LIB or load()).hatq_quantize_tokens(x.data_ptr(), kind, pitch, src_rows, index, n, c, hb, code, 1 if gated else 0,
                                               fmt, out.data_ptr(), out_pitch, ps, raw)
    if st:
        _check(st)
    return out, scales


def _product(x, scales, offsets, layer, dtype, out, stream):
    torch = _TORCH or _token_torch()
    device, raw = _launch_stream(x, stream)
    fmt, n, k, pitch = _rows_of(x, "x", _CODE_TYPES, device)
    if k != layer.k:
        raise ValueError(f"x: rows of {k} codes, the weights take {layer.k}")
    if pitch < k:
        x, pitch = _apart(x, stream), k
    if layer.device != device:
        raise ValueError(f"the weights are on cuda:{layer.device}, x on cuda:{device}")
    s_x = _flat(scales, "scales", torch.float32, (n,), device)
    if out is None:
        kind, out_pitch = _TOKEN_TYPES.get(dtype), layer.n
        if kind is None:
            raise ValueError(f"dtype {dtype} is none of {[str(d) for d in _TOKEN_TYPES]}")
        out = _empty(x, (n, out_pitch), dtype, stream)
    else:
        kind, out_pitch = _out_of(out, _TOKEN_TYPES, n, layer.n, device)
    lib, px = _LIB or load(), x.data_ptr()
    ws, size = None, 0
    if max(n, 32 * min(n, layer.experts)) * layer.size > 1_500_000_000 and not (
            fmt == CODES_F16 and pitch % 8 == 0 and px % 16 == 0):
        # More than about ten microseconds of products, or of weights to read: packing the codes may pay. Below, the
        # workspace and the second launch cost the host more than the GPU gains (777 rows, 1000 -> 1234: 20.6 us a
        # call with them, 12.6 us without).
        size = n * layer.row_bytes
        scratch = _empty(x, (size,), torch.uint8, stream)
        ws = scratch.data_ptr()
    if offsets is None:
        st = lib.hatq_linear(px, fmt, pitch, s_x, n, layer.ref, kind, out.data_ptr(), out_pitch, ws, size, raw)
    else:
        st = lib.hatq_grouped_linear(px, fmt, pitch, s_x, n,
                                     _flat(offsets, "offsets", torch.int32, (layer.experts + 1,), device), layer.ref,
                                     kind, out.data_ptr(), out_pitch, ws, size, raw)
    if st:
        _check(st)
    return out


def linear(x, scales, layer, dtype=None, out=None, stream=None):
    """hatq_linear: y [rows][n] of codes x [rows][k] (int8 or fp16) and their scales [rows],
    in `dtype` (float32, float16, bfloat16 - the default) or into `out`."""
    if layer.grouped:
        raise ValueError("a layer with experts needs grouped_linear")
    return _product(x, scales, None, layer, dtype or _token_torch().bfloat16, out, stream)


def grouped_linear(x, scales, offsets, layer, dtype=None, out=None, stream=None):
    """hatq_grouped_linear: rows offsets[e] .. offsets[e + 1] - 1 with expert e's weights
    (offsets int32 [experts + 1] on the device). Rows that no expert holds are not written."""
    if offsets is None:
        raise ValueError("offsets are missing")
    return _product(x, scales, offsets, layer, dtype or _token_torch().bfloat16, out, stream)


def combine_rows(y, index, weights, out=None, stream=None):
    """hatq_combine_rows: out[t] = sum_j weights[t][j] y[index[t][j]] (int32 index, float32 weights,
    both [tokens][topk]; an index outside y contributes nothing)."""
    torch = _TORCH or _token_torch()
    device, raw = _launch_stream(y, stream)
    kind, rows, c, pitch = _rows_of(y, "y", _TOKEN_TYPES, device)
    if pitch < c:
        y, pitch = _apart(y, stream), c
    if index.dim() != 2:
        raise ValueError(f"index: shape {tuple(index.shape)}, expected [tokens, topk]")
    t, topk = shape = index.shape
    if out is None:
        out, out_pitch = _empty(y, (t, c), y.dtype, stream), c
    else:
        out_kind, out_pitch = _out_of(out, _TOKEN_TYPES, t, c, device)
        if out_kind != kind:
            raise ValueError(f"out: {out.dtype}, expected {y.dtype}")
    st = (_LIB or load()).hatq_combine_rows(y.data_ptr(), kind, pitch, rows, _flat(index, "index", torch.int32, shape, device),
                                            _flat(weights, "weights", torch.float32, shape, device), t, topk, c,
                                            out.data_ptr(), out_pitch, raw)
    if st:
        _check(st)
    return out


# ------------------------------------------------------------------ the 4-bit cache

class TokenCache:
    """The 4-bit keys and values of one attention layer (hatq_token_cache): `data` is a contiguous uint8 CUDA tensor
    [pages][heads][page * (width + 8)] of the caller's, hb the block of the transform along a head."""

    def __init__(self, data, page=64, hb=1):
        torch = _token_torch()
        if data.dtype != torch.uint8 or data.dim() != 3 or not data.is_contiguous():
            raise ValueError("data: expected a contiguous uint8 tensor [pages][heads][page * (width + 8)]")
        pages, heads, size = data.shape
        if page not in (16, 32, 64) or size % page:
            raise ValueError(f"data: {size} bytes per head and page are no {page} tokens (16, 32 or 64 a page)")
        self.device = data.get_device()
        if self.device < 0:
            raise ValueError(f"expected CUDA tensors, got {data.device}")
        self.data, self.pages, self.page, self.heads, self.width, self.hb = data, pages, page, heads, size // page - 8, hb
        self.struct = TokenCacheStruct(data.data_ptr(), pages, page, heads, self.width, hb, 0)
        self.ref = ctypes.byref(self.struct)
        self.scale = self.width ** -0.5 if self.width > 0 else 1.0
        self.workspaces = {}                        # bytes of attend_tokens' workspace, by the sizes of a call
        size = ctypes.c_size_t()                    # the library looks the sizes over
        _check(load().hatq_attend_workspace(self.ref, BF16, heads, 0, 0, 0, 0, ctypes.byref(size)))

    @staticmethod
    def bytes_of(pages, heads, width, page=64):
        """Bytes of `data`: half a byte a value, and 8 bytes of scales per token and head."""
        return pages * heads * page * (width + 8)

    @classmethod
    def empty(cls, pages, heads, width, page=64, hb=None, device="cuda"):
        """A cache of its own memory; hb: by default the largest power of two that divides width."""
        torch = _torch()
        data = torch.empty(pages, heads, page * (width + 8), dtype=torch.uint8, device=device)
        return cls(data, page, (width & -width) if hb is None else hb)


def _heads_of(t, name, heads, width, device):
    """Checks a [rows][heads][width] tensor on `device` whose values are contiguous; returns its type code, its rows and
    the pitches of rows and heads in elements."""
    code = _TOKEN_TYPES.get(t.dtype)
    if code is None:
        raise ValueError(f"{name}: dtype {t.dtype} is none of {[str(d) for d in _TOKEN_TYPES]}")
    if t.dim() != 3 or heads and t.shape[1] != heads or t.shape[2] != width:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected [rows][{heads or 'heads'}][{width}]")
    if t.get_device() != device:
        raise ValueError(f"{name}: on {t.device}, expected cuda:{device}")
    pitch, head_pitch, inner = t.stride()
    if inner != 1:
        raise ValueError(f"{name}: the values of a head must be contiguous")
    return code, t.shape[0], pitch, head_pitch


def _sequences_of(table, lengths, starts, rows, device):
    """Checks the table [seqs][pages], lengths [seqs] and starts [seqs + 1] or None; returns what the library takes."""
    i32 = _TORCH.int32
    if table.dtype != i32 or table.dim() != 2 or table.get_device() != device:
        raise ValueError(f"table: expected an int32 tensor [sequences][pages] on cuda:{device}, got {table.dtype} "
                         f"{tuple(table.shape)} on {table.device}")
    seqs, width = table.shape
    pitch, inner = table.stride()
    if inner != 1 and width > 1:
        raise ValueError("table: the pages of a sequence must be contiguous")
    p = _flat(lengths, "lengths", i32, (seqs,), device)
    if starts is None:
        if rows != seqs:
            raise ValueError(f"{rows} rows for {seqs} sequences need starts")
        return table.data_ptr(), pitch, width, p, None, seqs
    return table.data_ptr(), pitch, width, p, _flat(starts, "starts", i32, (seqs + 1,), device), seqs


def append_tokens(cache, k, v, table, lengths, starts=None, kept=False, stream=None):
    """hatq_append_tokens: the newest tokens of every sequence into the cache.

    k, v [rows][heads][width]: sequence b has rows starts[b] .. starts[b + 1] - 1
    (starts int32 [sequences + 1]; None: one row each), its tokens up to
    lengths[b] - 1 (int32 [sequences], the new ones counted). table int32
    [sequences][pages]: token j lies in page table[b][j // cache.page]. All on the
    device and read there only. kept: also return (k, v) as the cache holds them
    now, in the inputs' type (rows that no sequence holds are not written)."""
    torch = _TORCH or _token_torch()
    device, raw = _launch_stream(k, stream)
    if cache.device != device:
        raise ValueError(f"the cache is on cuda:{cache.device}, k on cuda:{device}")
    heads, width = cache.heads, cache.width
    kind, rows, ldk, hk = _heads_of(k, "k", heads, width, device)
    v_kind, v_rows, ldv, hv = _heads_of(v, "v", heads, width, device)
    if v_kind != kind or v_rows != rows:
        raise ValueError(f"k and v differ: {k.dtype} {tuple(k.shape)}, {v.dtype} {tuple(v.shape)}")
    pt, ldt, pages, pl, ps, seqs = _sequences_of(table, lengths, starts, rows, device)
    out, pk, pv = None, None, None
    if kept:
        if stream is None and k.is_contiguous():
            out = torch.empty_like(k), torch.empty_like(k)
        else:
            out = _empty(k, k.shape, k.dtype, stream), _empty(k, k.shape, k.dtype, stream)
        pk, pv = out[0].data_ptr(), out[1].data_ptr()
    st = (_LIB or load()).hatq_append_tokens(cache.ref, k.data_ptr(), ldk, hk, v.data_ptr(), ldv, hv, kind, rows, pt, ldt,
                                             pages, pl, ps, seqs, pk, pv, raw)
    if st:
        _check(st)
    return out


def attend_tokens(q, cache, table, lengths, starts=None, scale=None, out=None, stream=None):
    """hatq_attend_tokens: causal softmax attention of q [rows][heads][width] (float16 or bfloat16) over the cache.

    Rows, table, lengths and starts as append_tokens takes them: a row sees its own
    token and those before it. The heads of q are a multiple of the cache's, those
    of one cache head next to each other. scale: width ** -0.5 unless given."""
    torch = _TORCH or _token_torch()
    device, raw = _launch_stream(q, stream)
    if cache.device != device:
        raise ValueError(f"the cache is on cuda:{cache.device}, q on cuda:{device}")
    kind, rows, ldq, hq = _heads_of(q, "q", 0, cache.width, device)
    heads = q.shape[1]
    pt, ldt, pages, pl, ps, seqs = _sequences_of(table, lengths, starts, rows, device)
    if out is None:
        out = torch.empty_like(q) if stream is None and q.is_contiguous() else _empty(q, q.shape, q.dtype, stream)
        ldo, ho = heads * cache.width, cache.width
    else:
        if out.dtype != q.dtype or out.shape != q.shape:
            raise ValueError(f"out: {out.dtype} {tuple(out.shape)}, expected {q.dtype} {tuple(q.shape)}")
        _, _, ldo, ho = _heads_of(out, "out", heads, cache.width, device)
    lib, sizes = _LIB or load(), (kind, heads, rows, seqs, pages, starts is None)
    size = cache.workspaces.get(sizes)
    if size is None:
        need = ctypes.c_size_t()
        _check(lib.hatq_attend_workspace(cache.ref, kind, heads, rows, seqs, 0 if starts is None else 1, pages, ctypes.byref(need)))
        if len(cache.workspaces) >= 256:
            cache.workspaces.clear()
        size = cache.workspaces[sizes] = need.value
    scratch = _empty(q, (size,), torch.uint8, stream) if size else None
    st = lib.hatq_attend_tokens(q.data_ptr(), kind, ldq, hq, heads, rows, cache.ref, pt, ldt, pages, pl, ps, seqs,
                                cache.scale if scale is None else scale, out.data_ptr(), ldo, ho,
                                scratch.data_ptr() if size else None, size, raw)
    if st:
        _check(st)
    return out


# ------------------------------------------------------------------ 4-bit weights

class Linear4Weights:
    """4-bit weights with one scale per group of inputs (hatq_linear4_weights): device buffers and the C struct."""

    def __init__(self, n, k, group, data, bias):
        self.n, self.k, self.group, self.data, self.bias = n, k, group, data, bias
        self.device = data.get_device()
        self.struct = Linear4WeightsStruct(n, k, group, 0, data.data_ptr(), None if bias is None else bias.data_ptr())
        self.ref = ctypes.byref(self.struct)


def quantize_groups(w, group=128, hb=1, stream=None):
    """hatq_quantize_groups: (codes int8 [n][k] in -7 .. 7, scales [n][groups]) of a floating-point matrix [n][k]."""
    torch = _TORCH or _token_torch()
    device, raw = _launch_stream(w, stream)
    kind, n, k, pitch = _rows_of(w, "w", _TOKEN_TYPES, device)
    if pitch < k:
        w, pitch = _apart(w, stream), k
    groups = -(-k // group) if group > 0 else 0
    codes, scales = _empty(w, (n, k), torch.int8, stream), _empty(w, (n, groups), torch.float32, stream)
    _check((_LIB or load()).hatq_quantize_groups(w.data_ptr(), kind, pitch, n, k, hb, group, codes.data_ptr(), k,
                                                 scales.data_ptr(), groups, raw))
    return codes, scales


def prepare_linear4(w, group=128, hb=1, scales=None, bias=None, stream=None) -> Linear4Weights:
    """The weights of linear4 (w [n][k]), on the device.

    w in float32 / float16 / bfloat16 (k <= 32768) is transformed along k in blocks
    of hb and quantized to 4 bits with one scale per output channel and `group`
    inputs (a multiple of 32; the last may be cut), as hatq_quantize_groups does;
    x must be transformed with the same hb (quantize_tokens does). w in int8 (-8 .. 7)
    is taken as it is, with `scales` [n][groups]. bias: [n], any floating type."""
    torch = _token_torch()
    _torch()
    if w.dim() != 2:
        raise ValueError(f"w: shape {tuple(w.shape)}, expected [n, k]")
    n, k = w.shape
    size = ctypes.c_size_t()
    _check(load().hatq_linear4_sizes(n, k, group, ctypes.byref(size)))
    device, raw = _launch_stream(w, stream)
    groups = -(-k // group)
    with torch.cuda.stream(stream):                 # None: the current one
        if w.dtype == torch.int8:
            if scales is None or hb != 1:
                raise ValueError("int8 weights need their scales, and are not transformed")
            if tuple(scales.shape) != (n, groups):
                raise ValueError(f"scales: shape {tuple(scales.shape)}, expected {(n, groups)}")
            codes, scales = w.contiguous(), scales.to(device=w.device, dtype=torch.float32).contiguous()
        else:
            if scales is not None:
                raise ValueError("scales belong to int8 weights")
            codes, scales = quantize_groups(w, group, hb, stream)
        if bias is not None:
            if bias.numel() != n:
                raise ValueError(f"bias: shape {tuple(bias.shape)}, expected {n} values")
            bias = bias.to(device=w.device, dtype=torch.float32).reshape(-1).clone()
        L = Linear4Weights(n, k, group, torch.empty(size.value, dtype=torch.uint8, device=w.device), bias)
        _check(load().hatq_linear4_layout(codes.data_ptr(), k, scales.data_ptr(), groups, L.ref, raw))
    return L


def linear4(x, layer, scales=None, dtype=None, out=None, stream=None):
    """hatq_linear4: y [rows][n] of x [rows][k] (float32, float16, bfloat16), in `dtype` (by default x's) or into `out`.

    scales: float32 [rows], a factor of each row: with x the "f16" codes of
    quantize_tokens, their scales."""
    torch = _TORCH or _token_torch()
    device, raw = _launch_stream(x, stream)
    x_kind, n, k, pitch = _rows_of(x, "x", _TOKEN_TYPES, device)
    if k != layer.k:
        raise ValueError(f"x: rows of {k} values, the weights take {layer.k}")
    if pitch < k:
        x, pitch = _apart(x, stream), k
    if layer.device != device:
        raise ValueError(f"the weights are on cuda:{layer.device}, x on cuda:{device}")
    s_x = None if scales is None else _flat(scales, "scales", torch.float32, (n,), device)
    if out is None:
        dtype = dtype or x.dtype
        kind, out_pitch = _TOKEN_TYPES.get(dtype), layer.n
        if kind is None:
            raise ValueError(f"dtype {dtype} is none of {[str(d) for d in _TOKEN_TYPES]}")
        out = _empty(x, (n, out_pitch), dtype, stream)
    else:
        kind, out_pitch = _out_of(out, _TOKEN_TYPES, n, layer.n, device)
    st = (_LIB or load()).hatq_linear4(x.data_ptr(), x_kind, pitch, s_x, n, layer.ref, kind, out.data_ptr(), out_pitch, raw)
    if st:
        _check(st)
    return out
