"""ctypes binding of the C-ABI library (include/gl.h): argument marshalling only.

Every function has the name of the C entry point it calls.  torch supplies
device memory and the current stream; nothing is computed in Python.  If the
shared library is missing, importing this module raises: there is no CPU path.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import Optional, Sequence

import torch

GL_MAX_DIMS = 8
GL_BF16, GL_F32 = 1, 2
GL_PAD_ZERO, GL_PAD_NEG_INF = 0, 1
GL_EPILOGUE_RELU = 0x2
GL_DOT_GENERAL_KERNEL = 0x100
GL_OUT_NCHW = 0x4
GL_OUT_BF16 = 0x8
GL_ROTATE_BACK = 0x10
GL_OK = 0

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libglenside.so")


class GlAp(ctypes.Structure):
    _fields_ = [
        ("data", ctypes.c_void_p),
        ("dtype", ctypes.c_int32),
        ("ndim", ctypes.c_int32),
        ("access_ndim", ctypes.c_int32),
        ("reserved_", ctypes.c_int32),
        ("shape", ctypes.c_int64 * GL_MAX_DIMS),
    ]


class GlWindows(ctypes.Structure):
    _fields_ = [
        ("n", ctypes.c_int32),
        ("pad_kind", ctypes.c_int32),
        ("wshape", ctypes.c_int64 * GL_MAX_DIMS),
        ("stride", ctypes.c_int64 * GL_MAX_DIMS),
        ("pad_lo", ctypes.c_int64 * GL_MAX_DIMS),
        ("pad_hi", ctypes.c_int64 * GL_MAX_DIMS),
    ]


class GlMx4(ctypes.Structure):
    _fields_ = [
        ("data", ctypes.c_void_p),
        ("scale", ctypes.c_void_p),
        ("ndim", ctypes.c_int32),
        ("access_ndim", ctypes.c_int32),
        ("shape", ctypes.c_int64 * GL_MAX_DIMS),
    ]


class GlCache4(ctypes.Structure):
    _fields_ = [
        ("data", ctypes.c_void_p),
        ("pages", ctypes.c_int64),
        ("kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("page_tokens", ctypes.c_int32),
        ("reserved_", ctypes.c_int32),
    ]


class GlPages(ctypes.Structure):
    _fields_ = [
        ("page_table", ctypes.c_void_p),
        ("lengths", ctypes.c_void_p),
        ("batch", ctypes.c_int32),
        ("table_width", ctypes.c_int32),
    ]


class GlF8(ctypes.Structure):
    _fields_ = list(GlMx4._fields_)


GL_MAX_PAIRS = 128


class GlRotary(ctypes.Structure):
    _fields_ = [
        ("pairs", ctypes.c_int32),
        ("axes", ctypes.c_int32),
        ("adjacent", ctypes.c_int32),
        ("reserved_", ctypes.c_int32),
        ("step", ctypes.c_uint64 * GL_MAX_PAIRS),
        ("axis", ctypes.c_uint8 * GL_MAX_PAIRS),
    ]


EXPORTS = [
    "gl_shape_access", "gl_shape_windows", "gl_shape_flatten", "gl_shape_transpose", "gl_shape_pad",
    "gl_shape_cartesian_dot", "gl_shape_reduce_max", "gl_access_windows", "gl_access_flatten",
    "gl_access_transpose", "gl_access_pad", "gl_cartesian_dot", "gl_cartesian_dot_workspace",
    "gl_compute_reduce_max", "gl_compute_relu", "gl_poll_device_status", "gl_strerror", "gl_version",
    "gl_cartesian_dot_static", "gl_shape_cartesian_dot_nchw",
    "gl_shape_slice", "gl_shape_concat", "gl_shape_pair", "gl_shape_squeeze", "gl_shape_reshape",
    "gl_shape_reduce_sum", "gl_access_slice", "gl_access_concat", "gl_access_pair", "gl_compute_reduce_sum",
    "gl_selftest_bounded_wait",
    "gl_mx4_data_bytes", "gl_mx4_scale_bytes", "gl_mx4_quantize", "gl_mx4_dequantize", "gl_cartesian_dot_mx4",
    "gl_dense_mx4", "gl_dense_mx4_workspace", "gl_cache4_bytes", "gl_cache4_append", "gl_cache4_read",
    "gl_attend_cache4", "gl_attend_cache4_workspace",
    "gl_f8_data_bytes", "gl_f8_scale_bytes", "gl_f8_quantize", "gl_f8_dequantize", "gl_cartesian_dot_f8", "gl_dense_f8",
    "gl_dense_f8_workspace", "gl_compute_norm_rms", "gl_compute_norm_rms_f8", "gl_rotary_plan", "gl_compute_rotate",
]


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            "libglenside.so is not built (run `python -m paper_2105_09377_b200.build`); "
            "there is no fallback path")
    lib = ctypes.CDLL(LIB_PATH)
    ap, win, vp = ctypes.POINTER(GlAp), ctypes.POINTER(GlWindows), ctypes.c_void_p
    i32p = ctypes.POINTER(ctypes.c_int32)
    mx, ca, pg = ctypes.POINTER(GlMx4), ctypes.POINTER(GlCache4), ctypes.POINTER(GlPages)
    f8, rot, f64p = ctypes.POINTER(GlF8), ctypes.POINTER(GlRotary), ctypes.POINTER(ctypes.c_double)
    sig = {
        "gl_shape_access": [ap, ctypes.c_int32, ap],
        "gl_shape_windows": [ap, win, ap],
        "gl_shape_flatten": [ap, ap],
        "gl_shape_transpose": [ap, i32p, ap],
        "gl_shape_pad": [ap, ctypes.c_int32, ctypes.c_int64, ctypes.c_int64, ap],
        "gl_shape_cartesian_dot": [ap, win, ap, ap],
        "gl_shape_cartesian_dot_nchw": [ap, win, ap, ap],
        "gl_shape_reduce_max": [ap, win, ap],
        "gl_shape_slice": [ap, ctypes.c_int32, ctypes.c_int64, ctypes.c_int64, ap],
        "gl_shape_concat": [ap, ap, ctypes.c_int32, ap],
        "gl_shape_pair": [ap, ap, ap],
        "gl_shape_squeeze": [ap, ctypes.c_int32, ap],
        "gl_shape_reshape": [ap, ctypes.POINTER(ctypes.c_int64), ctypes.c_int32, ctypes.c_int32, ap],
        "gl_shape_reduce_sum": [ap, ap],
        "gl_access_slice": [ap, ctypes.c_int32, ctypes.c_int64, ctypes.c_int64, ap, vp],
        "gl_access_concat": [ap, ap, ctypes.c_int32, ap, vp],
        "gl_access_pair": [ap, ap, ap, vp],
        "gl_compute_reduce_sum": [ap, ap, vp],
        "gl_access_windows": [ap, win, ap, vp],
        "gl_access_flatten": [ap, ap],
        "gl_access_transpose": [ap, i32p, ap, vp],
        "gl_access_pad": [ap, ctypes.c_int32, ctypes.c_int64, ctypes.c_int64, ctypes.c_int32, ap, vp],
        "gl_cartesian_dot": [ap, win, ap, ap, ctypes.c_uint32, vp, ctypes.c_size_t, vp],
        "gl_cartesian_dot_static": [ap, win, ap, ap, ctypes.c_uint32, vp],
        "gl_compute_reduce_max": [ap, win, ap, vp],
        "gl_compute_relu": [ap, ap, vp],
        "gl_poll_device_status": [vp],
        "gl_selftest_bounded_wait": [ctypes.c_uint32, vp],
        "gl_mx4_quantize": [ap, mx, vp],
        "gl_mx4_dequantize": [mx, ap, vp],
        "gl_cartesian_dot_mx4": [mx, mx, ap, ctypes.c_uint32, vp],
        "gl_dense_mx4": [ap, mx, ap, ctypes.c_uint32, vp, ctypes.c_size_t, vp],
        "gl_cache4_append": [ca, ap, ap, ctypes.c_int64, pg, vp],
        "gl_cache4_read": [ca, pg, ap, ap, vp],
        "gl_attend_cache4": [ap, ctypes.c_int64, ca, pg, ctypes.c_float, ap, ctypes.c_uint32, vp, ctypes.c_size_t, vp],
        "gl_f8_quantize": [ap, f8, vp],
        "gl_f8_dequantize": [f8, ap, vp],
        "gl_cartesian_dot_f8": [f8, f8, ap, ctypes.c_uint32, vp],
        "gl_dense_f8": [ap, f8, ap, ctypes.c_uint32, vp, ctypes.c_size_t, vp],
        "gl_compute_norm_rms": [ap, ap, ap, ctypes.c_float, ap, ap, vp],
        "gl_compute_norm_rms_f8": [ap, ap, ap, ctypes.c_float, ap, f8, vp],
        "gl_rotary_plan": [ctypes.c_int32, ctypes.c_double, f64p, i32p, ctypes.c_int32, ctypes.c_int32, rot],
        "gl_compute_rotate": [ap, ctypes.c_int64, rot, vp, ap, ctypes.c_int64, ctypes.c_uint32, vp],
    }
    for name, args in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = ctypes.c_int
    lib.gl_cartesian_dot_workspace.argtypes = [ap, win, ap, ctypes.c_uint32]
    lib.gl_cartesian_dot_workspace.restype = ctypes.c_size_t
    for name, args in {"gl_mx4_data_bytes": [mx], "gl_mx4_scale_bytes": [mx], "gl_dense_mx4_workspace": [ap, mx],
                       "gl_cache4_bytes": [ca], "gl_attend_cache4_workspace": [ap, ca],
                       "gl_f8_data_bytes": [f8], "gl_f8_scale_bytes": [f8], "gl_dense_f8_workspace": [ap, f8]}.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = ctypes.c_size_t
    lib.gl_strerror.argtypes = [ctypes.c_int]
    lib.gl_strerror.restype = ctypes.c_char_p
    lib.gl_version.restype = ctypes.c_int
    return lib


LIB = _load()
_BARE = ctypes.CDLL(LIB_PATH)   # the same library; its functions take C values as they are


class GlError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s: %s (code %d)" % (where, LIB.gl_strerror(code).decode(), code))


def _check(code: int, where: str):
    if code != GL_OK:
        raise GlError(code, where)


_DTYPES = {torch.bfloat16: GL_BF16, torch.float32: GL_F32}
_TORCH = {GL_BF16: torch.bfloat16, GL_F32: torch.float32}


@dataclass
class AccessPattern:
    """A dense device tensor viewed as (access dims, compute dims)."""

    tensor: torch.Tensor
    access_ndim: int

    @property
    def access_shape(self):
        return tuple(self.tensor.shape[: self.access_ndim])

    @property
    def compute_shape(self):
        return tuple(self.tensor.shape[self.access_ndim:])

    @property
    def shape(self):
        return (self.access_shape, self.compute_shape)


def _meta(shape: Sequence[int], access_ndim: int, dtype: int, data: int = 0) -> GlAp:
    if len(shape) > GL_MAX_DIMS:
        raise GlError(3, "too many dimensions")
    m = GlAp()
    m.data = data
    m.dtype = dtype
    m.ndim = len(shape)
    m.access_ndim = access_ndim
    for i, s in enumerate(shape):
        m.shape[i] = int(s)
    return m


def _struct(a: AccessPattern) -> GlAp:
    t = a.tensor
    if not t.is_contiguous():
        raise ValueError("access patterns are dense row-major tensors")
    return _meta(tuple(t.shape), a.access_ndim, _DTYPES[t.dtype], t.data_ptr())


def _stream_object(stream):
    """`stream` as torch knows it: a torch stream, or the address of one of another library (0: the default stream)."""
    if hasattr(stream, "cuda_stream"):
        return stream
    return torch.cuda.ExternalStream(int(stream)) if int(stream) else torch.cuda.default_stream()


def _empty(shape, dtype, device, stream) -> torch.Tensor:
    """Storage that the call on `stream` (None: the current one) writes.  torch hands a block out again as soon as its tensor
    is gone, in the order of the stream that it was taken on: so it is taken on the stream that the call runs on, and scratch
    may be dropped when the call returns."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(_stream_object(stream)):
        return torch.empty(shape, dtype=dtype, device=device)


def _scratch(need: int, device, stream=None) -> Optional[torch.Tensor]:
    return _empty(need + 1024, torch.uint8, device, stream) if need else None


def _alloc(meta: GlAp, device, stream=None) -> AccessPattern:
    shape = tuple(meta.shape[i] for i in range(meta.ndim))
    return AccessPattern(_empty(shape, _TORCH[meta.dtype], device, stream), meta.access_ndim)


def _stream(stream) -> int:
    if stream is None:
        # torch.cuda.current_stream() builds a Stream object: 3.3 us, next to 2 us for a kernel launch
        torch.cuda.is_initialized() or torch.cuda.init()
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def windows_spec(wshape, stride, pad_lo=None, pad_hi=None, pad_kind=GL_PAD_ZERO) -> GlWindows:
    n = len(wshape)
    w = GlWindows()
    w.n = n
    w.pad_kind = pad_kind
    pad_lo = pad_lo or [0] * n
    pad_hi = pad_hi or [0] * n
    for i in range(n):
        w.wshape[i], w.stride[i], w.pad_lo[i], w.pad_hi[i] = int(wshape[i]), int(stride[i]), int(pad_lo[i]), int(pad_hi[i])
    return w


def _wptr(w: Optional[GlWindows]):
    return ctypes.byref(w) if w is not None else None


# ---- host-only shape inference: (shape, access_ndim, dtype) in, the same out ----

def _shape_result(m: GlAp):
    return tuple(m.shape[i] for i in range(m.ndim)), m.access_ndim, m.dtype


def gl_shape_access(shape, access_ndim, i, dtype=GL_F32):
    out = GlAp()
    _check(LIB.gl_shape_access(ctypes.byref(_meta(shape, access_ndim, dtype)), i, ctypes.byref(out)), "gl_shape_access")
    return _shape_result(out)


def gl_shape_windows(shape, access_ndim, w: GlWindows, dtype=GL_F32):
    out = GlAp()
    _check(LIB.gl_shape_windows(ctypes.byref(_meta(shape, access_ndim, dtype)), ctypes.byref(w), ctypes.byref(out)),
           "gl_shape_windows")
    return _shape_result(out)


def gl_shape_flatten(shape, access_ndim, dtype=GL_F32):
    out = GlAp()
    _check(LIB.gl_shape_flatten(ctypes.byref(_meta(shape, access_ndim, dtype)), ctypes.byref(out)), "gl_shape_flatten")
    return _shape_result(out)


def gl_shape_transpose(shape, access_ndim, perm, dtype=GL_F32):
    out = GlAp()
    arr = (ctypes.c_int32 * len(perm))(*perm)
    _check(LIB.gl_shape_transpose(ctypes.byref(_meta(shape, access_ndim, dtype)), arr, ctypes.byref(out)),
           "gl_shape_transpose")
    return _shape_result(out)


def gl_shape_pad(shape, access_ndim, dim, lo, hi, dtype=GL_F32):
    out = GlAp()
    _check(LIB.gl_shape_pad(ctypes.byref(_meta(shape, access_ndim, dtype)), dim, lo, hi, ctypes.byref(out)), "gl_shape_pad")
    return _shape_result(out)


def gl_shape_cartesian_dot(shape0, access0, w: Optional[GlWindows], shape1, access1):
    out = GlAp()
    _check(LIB.gl_shape_cartesian_dot(ctypes.byref(_meta(shape0, access0, GL_BF16)), _wptr(w),
                                      ctypes.byref(_meta(shape1, access1, GL_BF16)), ctypes.byref(out)),
           "gl_shape_cartesian_dot")
    return _shape_result(out)


def gl_shape_cartesian_dot_nchw(shape0, access0, w: GlWindows, shape1, access1):
    out = GlAp()
    _check(LIB.gl_shape_cartesian_dot_nchw(ctypes.byref(_meta(shape0, access0, GL_BF16)), ctypes.byref(w),
                                           ctypes.byref(_meta(shape1, access1, GL_BF16)), ctypes.byref(out)),
           "gl_shape_cartesian_dot_nchw")
    return _shape_result(out)


def gl_shape_reduce_max(shape, access_ndim, w: Optional[GlWindows]):
    out = GlAp()
    _check(LIB.gl_shape_reduce_max(ctypes.byref(_meta(shape, access_ndim, GL_F32)), _wptr(w), ctypes.byref(out)),
           "gl_shape_reduce_max")
    return _shape_result(out)


# ---- device operations ----

def gl_access_windows(a: AccessPattern, w: GlWindows, out: Optional[AccessPattern] = None, stream=None) -> AccessPattern:
    sa = _struct(a)
    if out is None:
        m = GlAp()
        _check(LIB.gl_shape_windows(ctypes.byref(sa), ctypes.byref(w), ctypes.byref(m)), "gl_shape_windows")
        out = _alloc(m, a.tensor.device, stream)
    so = _struct(out)
    _check(LIB.gl_access_windows(ctypes.byref(sa), ctypes.byref(w), ctypes.byref(so), _stream(stream)), "gl_access_windows")
    return out


def gl_access_flatten(a: AccessPattern) -> AccessPattern:
    sa, so = _struct(a), GlAp()
    _check(LIB.gl_access_flatten(ctypes.byref(sa), ctypes.byref(so)), "gl_access_flatten")
    assert so.data == sa.data
    shape = tuple(so.shape[i] for i in range(so.ndim))
    return AccessPattern(a.tensor.view(shape), so.access_ndim)


def gl_access_transpose(a: AccessPattern, perm, out: Optional[AccessPattern] = None, stream=None) -> AccessPattern:
    sa = _struct(a)
    arr = (ctypes.c_int32 * len(perm))(*perm)
    if out is None:
        m = GlAp()
        _check(LIB.gl_shape_transpose(ctypes.byref(sa), arr, ctypes.byref(m)), "gl_shape_transpose")
        out = _alloc(m, a.tensor.device, stream)
    so = _struct(out)
    _check(LIB.gl_access_transpose(ctypes.byref(sa), arr, ctypes.byref(so), _stream(stream)), "gl_access_transpose")
    return out


def gl_access_pad(a: AccessPattern, dim: int, lo: int, hi: int, pad_kind=GL_PAD_ZERO,
                  out: Optional[AccessPattern] = None, stream=None) -> AccessPattern:
    sa = _struct(a)
    if out is None:
        m = GlAp()
        _check(LIB.gl_shape_pad(ctypes.byref(sa), dim, lo, hi, ctypes.byref(m)), "gl_shape_pad")
        out = _alloc(m, a.tensor.device, stream)
    so = _struct(out)
    _check(LIB.gl_access_pad(ctypes.byref(sa), dim, lo, hi, pad_kind, ctypes.byref(so), _stream(stream)), "gl_access_pad")
    return out


def gl_cartesian_dot_workspace(a0: AccessPattern, w: Optional[GlWindows], a1: AccessPattern, flags: int = 0) -> int:
    return int(LIB.gl_cartesian_dot_workspace(ctypes.byref(_struct(a0)), _wptr(w), ctypes.byref(_struct(a1)), flags))


def gl_cartesian_dot(a0: AccessPattern, w: Optional[GlWindows], a1: AccessPattern, out: Optional[AccessPattern] = None,
                     flags: int = 0, workspace: Optional[torch.Tensor] = None, stream=None) -> AccessPattern:
    s0, s1 = _struct(a0), _struct(a1)
    if out is None:
        m = GlAp()
        if flags & GL_OUT_NCHW:
            _check(LIB.gl_shape_cartesian_dot_nchw(ctypes.byref(s0), _wptr(w), ctypes.byref(s1), ctypes.byref(m)),
                   "gl_shape_cartesian_dot_nchw")
        else:
            _check(LIB.gl_shape_cartesian_dot(ctypes.byref(s0), _wptr(w), ctypes.byref(s1), ctypes.byref(m)),
                   "gl_shape_cartesian_dot")
        if flags & GL_OUT_BF16:
            m.dtype = GL_BF16
        out = _alloc(m, a0.tensor.device, stream)
    if workspace is None:
        need = int(LIB.gl_cartesian_dot_workspace(ctypes.byref(s0), _wptr(w), ctypes.byref(s1), flags))
        if need:
            workspace = _scratch(need, a0.tensor.device, stream)
    ws_ptr, ws_bytes = 0, 0
    if workspace is not None:
        ws_ptr = (workspace.data_ptr() + 1023) // 1024 * 1024
        ws_bytes = workspace.numel() * workspace.element_size() - (ws_ptr - workspace.data_ptr())
    so = _struct(out)
    _check(LIB.gl_cartesian_dot(ctypes.byref(s0), _wptr(w), ctypes.byref(s1), ctypes.byref(so), flags, ws_ptr, ws_bytes,
                                _stream(stream)), "gl_cartesian_dot")
    return out


GL_STATIC_SCRATCH_BYTES = 32 << 20


def gl_cartesian_dot_static(a0: AccessPattern, w: Optional[GlWindows], a1: AccessPattern, out: AccessPattern,
                            flags: int = 0, stream=None) -> AccessPattern:
    """gl_cartesian_dot without a workspace argument, for callers that may not allocate device
    memory: the scratch is a fixed 32 MiB array inside the library.  `out` must be supplied (this
    wrapper allocates nothing either).  Calls that may overlap on the GPU must be ordered by the
    caller, and the first call on a device should precede any stream capture."""
    s0, s1, so = _struct(a0), _struct(a1), _struct(out)
    _check(LIB.gl_cartesian_dot_static(ctypes.byref(s0), _wptr(w), ctypes.byref(s1), ctypes.byref(so), flags,
                                       _stream(stream)), "gl_cartesian_dot_static")
    return out


def gl_compute_reduce_max(a: AccessPattern, w: Optional[GlWindows], out: Optional[AccessPattern] = None,
                          stream=None) -> AccessPattern:
    sa = _struct(a)
    if out is None:
        m = GlAp()
        _check(LIB.gl_shape_reduce_max(ctypes.byref(sa), _wptr(w), ctypes.byref(m)), "gl_shape_reduce_max")
        out = _alloc(m, a.tensor.device, stream)
    so = _struct(out)
    _check(LIB.gl_compute_reduce_max(ctypes.byref(sa), _wptr(w), ctypes.byref(so), _stream(stream)), "gl_compute_reduce_max")
    return out


def gl_access_slice(a: AccessPattern, dim: int, lo: int, hi: int, out: Optional[AccessPattern] = None,
                    stream=None) -> AccessPattern:
    sa = _struct(a)
    if out is None:
        m = GlAp()
        _check(LIB.gl_shape_slice(ctypes.byref(sa), dim, lo, hi, ctypes.byref(m)), "gl_shape_slice")
        out = _alloc(m, a.tensor.device, stream)
    so = _struct(out)
    _check(LIB.gl_access_slice(ctypes.byref(sa), dim, lo, hi, ctypes.byref(so), _stream(stream)), "gl_access_slice")
    return out


def gl_access_concat(a: AccessPattern, b: AccessPattern, dim: int, out: Optional[AccessPattern] = None,
                     stream=None) -> AccessPattern:
    sa, sb = _struct(a), _struct(b)
    if out is None:
        m = GlAp()
        _check(LIB.gl_shape_concat(ctypes.byref(sa), ctypes.byref(sb), dim, ctypes.byref(m)), "gl_shape_concat")
        out = _alloc(m, a.tensor.device, stream)
    so = _struct(out)
    _check(LIB.gl_access_concat(ctypes.byref(sa), ctypes.byref(sb), dim, ctypes.byref(so), _stream(stream)),
           "gl_access_concat")
    return out


def gl_access_pair(a: AccessPattern, b: AccessPattern, out: Optional[AccessPattern] = None, stream=None) -> AccessPattern:
    sa, sb = _struct(a), _struct(b)
    if out is None:
        m = GlAp()
        _check(LIB.gl_shape_pair(ctypes.byref(sa), ctypes.byref(sb), ctypes.byref(m)), "gl_shape_pair")
        out = _alloc(m, a.tensor.device, stream)
    so = _struct(out)
    _check(LIB.gl_access_pair(ctypes.byref(sa), ctypes.byref(sb), ctypes.byref(so), _stream(stream)), "gl_access_pair")
    return out


def gl_access_squeeze(a: AccessPattern, dim: int) -> AccessPattern:
    """`squeeze` is metadata: the result views the same storage."""
    m = GlAp()
    _check(LIB.gl_shape_squeeze(ctypes.byref(_struct(a)), dim, ctypes.byref(m)), "gl_shape_squeeze")
    return AccessPattern(a.tensor.view(tuple(m.shape[i] for i in range(m.ndim))), m.access_ndim)


def gl_access_reshape(a: AccessPattern, access_shape, compute_shape) -> AccessPattern:
    """`reshape` is metadata: the result views the same storage."""
    shape = tuple(access_shape) + tuple(compute_shape)
    arr = (ctypes.c_int64 * max(1, len(shape)))(*shape)
    m = GlAp()
    _check(LIB.gl_shape_reshape(ctypes.byref(_struct(a)), arr, len(shape), len(access_shape), ctypes.byref(m)),
           "gl_shape_reshape")
    return AccessPattern(a.tensor.view(shape), len(access_shape))


def gl_compute_reduce_sum(a: AccessPattern, out: Optional[AccessPattern] = None, stream=None) -> AccessPattern:
    sa = _struct(a)
    if out is None:
        m = GlAp()
        _check(LIB.gl_shape_reduce_sum(ctypes.byref(sa), ctypes.byref(m)), "gl_shape_reduce_sum")
        out = _alloc(m, a.tensor.device, stream)
    so = _struct(out)
    _check(LIB.gl_compute_reduce_sum(ctypes.byref(sa), ctypes.byref(so), _stream(stream)), "gl_compute_reduce_sum")
    return out


def gl_compute_relu(a: AccessPattern, out: Optional[AccessPattern] = None, stream=None) -> AccessPattern:
    sa = _struct(a)
    if out is None:
        out = AccessPattern(_empty(a.tensor.shape, a.tensor.dtype, a.tensor.device, stream), a.access_ndim)
    so = _struct(out)
    _check(LIB.gl_compute_relu(ctypes.byref(sa), ctypes.byref(so), _stream(stream)), "gl_compute_relu")
    return out


# ---- operands held in 4 bits ----

def _on_gpu(*tensors):
    """The kernels read these addresses themselves: a tensor on the host (lengths or a page table made there, say) would be
    a fault of the GPU."""
    device = tensors[0].device
    for t in tensors:
        if t is not None and not (t.is_cuda and t.device == device):
            raise ValueError("tensors have to be on one GPU: %s and %s" % (device, t.device))


@dataclass
class Mx4:
    """A pattern held in 4 bits: E2M1 codes (two a byte) and one E8M0 scale per 32 values of an item."""

    data: torch.Tensor    # uint8, gl_mx4_data_bytes
    scale: torch.Tensor   # uint8, gl_mx4_scale_bytes
    dims: tuple           # S_A ++ S_C
    access_ndim: int

    @property
    def shape(self):
        return (self.dims[: self.access_ndim], self.dims[self.access_ndim:])


def _mx4_struct(m: Mx4) -> GlMx4:
    s = _mx4_meta(m.dims, m.access_ndim)
    for t, need in ((m.data, LIB.gl_mx4_data_bytes(ctypes.byref(s))), (m.scale, LIB.gl_mx4_scale_bytes(ctypes.byref(s)))):
        if t.dtype != torch.uint8 or not t.is_contiguous() or t.numel() < need:
            raise ValueError("an MX4 operand of this shape wants %d contiguous bytes" % need)
    s.data, s.scale = m.data.data_ptr(), m.scale.data_ptr()
    return s


def _mx4_meta(shape, access_ndim) -> GlMx4:
    if len(shape) > GL_MAX_DIMS:
        raise GlError(3, "too many dimensions")
    s = GlMx4()
    s.ndim, s.access_ndim = len(shape), access_ndim
    for i, n in enumerate(shape):
        s.shape[i] = int(n)
    return s


def mx4_empty(shape, access_ndim: int, device, stream=None) -> Mx4:
    """Storage for a pattern of this shape, contents undefined; `stream`: where it is first used, if not the current one."""
    s = _mx4_meta(shape, access_ndim)
    nd, ns = LIB.gl_mx4_data_bytes(ctypes.byref(s)), LIB.gl_mx4_scale_bytes(ctypes.byref(s))
    if not nd:
        raise GlError(4, "mx4_empty")
    return Mx4(_empty(nd, torch.uint8, device, stream), _empty(ns, torch.uint8, device, stream),
               tuple(int(n) for n in shape), access_ndim)


def gl_mx4_quantize(a: AccessPattern, out: Optional[Mx4] = None, stream=None) -> Mx4:
    sa = _struct(a)
    if out is None:
        out = mx4_empty(tuple(a.tensor.shape), a.access_ndim, a.tensor.device, stream)
    _on_gpu(a.tensor, out.data, out.scale)
    _check(LIB.gl_mx4_quantize(ctypes.byref(sa), ctypes.byref(_mx4_struct(out)), _stream(stream)), "gl_mx4_quantize")
    return out


def gl_mx4_dequantize(m: Mx4, out: Optional[AccessPattern] = None, stream=None) -> AccessPattern:
    if out is None:
        out = AccessPattern(_empty(m.dims, torch.float32, m.data.device, stream), m.access_ndim)
    _on_gpu(m.data, m.scale, out.tensor)
    so = _struct(out)
    _check(LIB.gl_mx4_dequantize(ctypes.byref(_mx4_struct(m)), ctypes.byref(so), _stream(stream)), "gl_mx4_dequantize")
    return out


def _product_out(access0, access1, flags, device, stream) -> AccessPattern:
    shape = tuple(access0) + tuple(access1)
    dtype = torch.bfloat16 if flags & GL_OUT_BF16 else torch.float32
    return AccessPattern(_empty(shape, dtype, device, stream), len(shape))


def gl_cartesian_dot_mx4(a0: Mx4, a1: Mx4, out: Optional[AccessPattern] = None, flags: int = 0, stream=None) -> AccessPattern:
    if out is None:
        out = _product_out(a0.shape[0], a1.shape[0], flags, a0.data.device, stream)
    _on_gpu(a0.data, a0.scale, a1.data, a1.scale, out.tensor)
    so = _struct(out)
    _check(LIB.gl_cartesian_dot_mx4(ctypes.byref(_mx4_struct(a0)), ctypes.byref(_mx4_struct(a1)), ctypes.byref(so), flags,
                                    _stream(stream)), "gl_cartesian_dot_mx4")
    return out


def gl_dense_mx4_workspace(a0: AccessPattern, a1: Mx4) -> int:
    return int(LIB.gl_dense_mx4_workspace(ctypes.byref(_struct(a0)), ctypes.byref(_mx4_struct(a1))))


def gl_dense_mx4(a0: AccessPattern, a1: Mx4, out: Optional[AccessPattern] = None, flags: int = 0,
                 workspace: Optional[torch.Tensor] = None, stream=None) -> AccessPattern:
    if out is None:
        out = _product_out(a0.access_shape, a1.shape[0], flags, a0.tensor.device, stream)
    if workspace is None:
        workspace = _scratch(gl_dense_mx4_workspace(a0, a1), a0.tensor.device, stream)
    _on_gpu(a0.tensor, a1.data, a1.scale, out.tensor, workspace)
    s0, so = _struct(a0), _struct(out)
    _check(LIB.gl_dense_mx4(ctypes.byref(s0), ctypes.byref(_mx4_struct(a1)), ctypes.byref(so), flags, *_ws(workspace),
                            _stream(stream)), "gl_dense_mx4")
    return out


# ---- operands held in 8 bits, the norm in front of them ----

def _on_this_gpu(*tensors) -> int:
    """`_on_gpu`, and that GPU is the current one, whose streams and kernels the library uses; returns its index."""
    _on_gpu(*tensors)
    return _current_is(tensors[0].device.index)


def _current_is(index: int) -> int:
    if torch._C._cuda_getDevice() != index:
        raise ValueError("tensors are on GPU %d, which is not the current one: call under torch.cuda.device" % index)
    return index


@dataclass
class F8:
    """A pattern held in 8 bits: E4M3 codes and one E8M0 scale per 128 values of an item."""

    data: torch.Tensor    # uint8, gl_f8_data_bytes
    scale: torch.Tensor   # uint8, gl_f8_scale_bytes
    dims: tuple           # S_A ++ S_C
    access_ndim: int

    @property
    def shape(self):
        return (self.dims[: self.access_ndim], self.dims[self.access_ndim:])


def _f8_meta(shape, access_ndim) -> GlF8:
    if len(shape) > GL_MAX_DIMS:
        raise GlError(3, "too many dimensions")
    s = GlF8()
    s.ndim, s.access_ndim = len(shape), access_ndim
    for i, n in enumerate(shape):
        s.shape[i] = int(n)
    return s


def _f8_struct(m: F8) -> GlF8:
    s = _f8_meta(m.dims, m.access_ndim)
    for t, need in ((m.data, LIB.gl_f8_data_bytes(ctypes.byref(s))), (m.scale, LIB.gl_f8_scale_bytes(ctypes.byref(s)))):
        if t.dtype != torch.uint8 or not t.is_contiguous() or t.numel() < need:
            raise ValueError("an F8 operand of this shape wants %d contiguous bytes" % need)
    s.data, s.scale = m.data.data_ptr(), m.scale.data_ptr()
    return s


def f8_empty(shape, access_ndim: int, device, stream=None) -> F8:
    """Storage for a pattern of this shape, contents undefined; `stream`: where it is first used, if not the current one."""
    s = _f8_meta(shape, access_ndim)
    nd, ns = LIB.gl_f8_data_bytes(ctypes.byref(s)), LIB.gl_f8_scale_bytes(ctypes.byref(s))
    if not nd:
        raise GlError(4, "f8_empty")
    return F8(_empty(nd, torch.uint8, device, stream), _empty(ns, torch.uint8, device, stream),
              tuple(int(n) for n in shape), access_ndim)


def gl_f8_quantize(a: AccessPattern, out: Optional[F8] = None, stream=None) -> F8:
    sa = _struct(a)
    if out is None:
        out = f8_empty(tuple(a.tensor.shape), a.access_ndim, a.tensor.device, stream)
    _on_this_gpu(a.tensor, out.data, out.scale)
    _check(LIB.gl_f8_quantize(ctypes.byref(sa), ctypes.byref(_f8_struct(out)), _stream(stream)), "gl_f8_quantize")
    return out


def gl_f8_dequantize(m: F8, out: Optional[AccessPattern] = None, stream=None) -> AccessPattern:
    if out is None:
        out = AccessPattern(_empty(m.dims, torch.float32, m.data.device, stream), m.access_ndim)
    _on_this_gpu(m.data, m.scale, out.tensor)
    so = _struct(out)
    _check(LIB.gl_f8_dequantize(ctypes.byref(_f8_struct(m)), ctypes.byref(so), _stream(stream)), "gl_f8_dequantize")
    return out


def gl_cartesian_dot_f8(a0: F8, a1: F8, out: Optional[AccessPattern] = None, flags: int = 0, stream=None) -> AccessPattern:
    if out is None:
        out = _product_out(a0.shape[0], a1.shape[0], flags, a0.data.device, stream)
    _on_this_gpu(a0.data, a0.scale, a1.data, a1.scale, out.tensor)
    so = _struct(out)
    _check(LIB.gl_cartesian_dot_f8(ctypes.byref(_f8_struct(a0)), ctypes.byref(_f8_struct(a1)), ctypes.byref(so), flags,
                                   _stream(stream)), "gl_cartesian_dot_f8")
    return out


def gl_dense_f8_workspace(a0: AccessPattern, a1: F8) -> int:
    return int(LIB.gl_dense_f8_workspace(ctypes.byref(_struct(a0)), ctypes.byref(_f8_struct(a1))))


def gl_dense_f8(a0: AccessPattern, a1: F8, out: Optional[AccessPattern] = None, flags: int = 0,
                workspace: Optional[torch.Tensor] = None, stream=None) -> AccessPattern:
    if out is None:
        out = _product_out(a0.access_shape, a1.shape[0], flags, a0.tensor.device, stream)
    if workspace is None:
        workspace = _scratch(gl_dense_f8_workspace(a0, a1), a0.tensor.device, stream)
    _on_this_gpu(a0.tensor, a1.data, a1.scale, out.tensor, workspace)
    s0, so = _struct(a0), _struct(out)
    _check(LIB.gl_dense_f8(ctypes.byref(s0), ctypes.byref(_f8_struct(a1)), ctypes.byref(so), flags, *_ws(workspace),
                           _stream(stream)), "gl_dense_f8")
    return out


def _ap_ptr(a: Optional[AccessPattern]):
    return ctypes.byref(_struct(a)) if a is not None else None


def _tensor(a: Optional[AccessPattern]):
    return a.tensor if a is not None else None


def _norm_call(x, weight, out, eps, residual, total):
    """(entry point, arguments) of a norm whose result is an F8 operand or an access pattern."""
    eight = isinstance(out, F8)
    _on_this_gpu(x.tensor, _tensor(weight), _tensor(residual), _tensor(total), *((out.data, out.scale) if eight else (out.tensor,)))
    args = (_ap_ptr(x), _ap_ptr(residual), _ap_ptr(weight), float(eps), _ap_ptr(total),
            ctypes.byref(_f8_struct(out)) if eight else _ap_ptr(out))
    return (LIB.gl_compute_norm_rms_f8 if eight else LIB.gl_compute_norm_rms), args


def gl_compute_norm_rms(x: AccessPattern, weight: Optional[AccessPattern] = None, eps: float = 1e-6,
                        residual: Optional[AccessPattern] = None, total: Optional[AccessPattern] = None, out=None, stream=None):
    """`out`: an access pattern of x's shape (default: of x's type) or an F8 operand, whose storage says where the result goes.
    `total` takes x + residual in the residual's type (the header's `sum`); it may be `residual`."""
    if out is None:
        out = AccessPattern(_empty(tuple(x.tensor.shape), x.tensor.dtype, x.tensor.device, stream), x.access_ndim)
    call, args = _norm_call(x, weight, out, eps, residual, total)
    _check(call(*args, _stream(stream)), call.__name__)
    return out


def gl_compute_norm_rms_f8(x: AccessPattern, weight: Optional[AccessPattern] = None, eps: float = 1e-6,
                           residual: Optional[AccessPattern] = None, total: Optional[AccessPattern] = None,
                           out: Optional[F8] = None, stream=None) -> F8:
    if out is None:
        out = f8_empty(tuple(x.tensor.shape), x.access_ndim, x.tensor.device, stream)
    return gl_compute_norm_rms(x, weight, eps, residual, total, out, stream)


# ---- rotary positions ----

def rotary_plan(pairs: int, base: float = 10000.0, sections: Optional[Sequence[int]] = None, adjacent: bool = False,
                freq: Optional[Sequence[float]] = None) -> GlRotary:
    """Frequencies base^(-i / pairs), or `freq` (radians per position), `sections`: consecutive pairs of each axis."""
    if freq is not None and len(freq) != pairs:
        raise ValueError("one frequency per pair")
    sections = [pairs] if sections is None else list(sections)
    plan = GlRotary()
    _check(LIB.gl_rotary_plan(pairs, float(base), (ctypes.c_double * pairs)(*freq) if freq is not None else None,
                              (ctypes.c_int32 * max(1, len(sections)))(*sections), len(sections), int(adjacent),
                              ctypes.byref(plan)), "gl_rotary_plan")
    return plan


def _rotate_args(x: AccessPattern, plan: GlRotary, positions: torch.Tensor, out: AccessPattern, flags: int):
    _on_this_gpu(x.tensor, positions, out.tensor)
    sx, pitch = _tokens_struct(x.tensor)
    so, out_pitch = _tokens_struct(out.tensor)
    sx.access_ndim, so.access_ndim = x.access_ndim, out.access_ndim
    batch_tokens = tuple(x.tensor.shape[:2])
    shapes = [(plan.axes,) + batch_tokens] + ([batch_tokens] if plan.axes == 1 else [])
    if positions.dtype != torch.int32 or not positions.is_contiguous() or tuple(positions.shape) not in shapes:
        raise ValueError("positions are contiguous int32 [axes, batch, tokens]")
    # (a copy: what the caller changes in the plan later has not been checked against these positions)
    return (ctypes.byref(sx), pitch, ctypes.byref(GlRotary.from_buffer_copy(plan)), positions.data_ptr(), ctypes.byref(so), out_pitch, flags)


def gl_compute_rotate(x: AccessPattern, plan: GlRotary, positions: torch.Tensor, out: Optional[AccessPattern] = None, flags: int = 0,
                      stream=None) -> AccessPattern:
    """x ((B, T, heads),(head_dim)), whose tokens may lie further apart than they are long; positions int32 [axes, B, T], or
    [B, T] with one axis; out may be x."""
    if out is None:
        out = AccessPattern(_empty(tuple(x.tensor.shape), x.tensor.dtype, x.tensor.device, stream), 3)
    _check(LIB.gl_compute_rotate(*_rotate_args(x, plan, positions, out, flags), _stream(stream)), "gl_compute_rotate")
    return out


# ---- pages of 4-bit keys and values ----

@dataclass
class Cache4:
    """Pages of keys and values held in 4 bits; the order of the bytes is the library's own."""

    data: torch.Tensor    # uint8, gl_cache4_bytes
    pages: int
    kv_heads: int
    page_tokens: int
    head_dim: int


def _cache4_struct(c: Cache4) -> GlCache4:
    s = GlCache4()
    s.data, s.pages, s.kv_heads, s.head_dim, s.page_tokens = 0, c.pages, c.kv_heads, c.head_dim, c.page_tokens
    if c.data is not None:
        if c.data.dtype != torch.uint8 or not c.data.is_contiguous() or c.data.numel() < LIB.gl_cache4_bytes(ctypes.byref(s)):
            raise ValueError("the cache's storage is smaller than gl_cache4_bytes, or not contiguous bytes")
        s.data = c.data.data_ptr()
    return s


def cache4_empty(pages: int, kv_heads: int, page_tokens: int, head_dim: int, device) -> Cache4:
    """Storage for `pages` pages, contents undefined (a token is readable once it has been appended)."""
    c = Cache4(None, pages, kv_heads, page_tokens, head_dim)
    need = LIB.gl_cache4_bytes(ctypes.byref(_cache4_struct(c)))
    if not need:
        raise GlError(7, "cache4_empty")
    c.data = torch.empty(need, dtype=torch.uint8, device=device)
    return c


def _pages_struct(page_table: torch.Tensor, lengths: torch.Tensor) -> GlPages:
    if page_table.dtype != torch.int32 or lengths.dtype != torch.int32 or page_table.dim() != 2 or lengths.dim() != 1:
        raise ValueError("page_table is int32 [batch, width] and lengths int32 [batch]")
    if not page_table.is_contiguous() or not lengths.is_contiguous() or page_table.shape[0] != lengths.shape[0]:
        raise ValueError("page_table and lengths are contiguous and agree in the batch")
    s = GlPages()
    s.page_table, s.lengths = page_table.data_ptr(), lengths.data_ptr()
    s.batch, s.table_width = page_table.shape
    return s


def _tokens_struct(t: torch.Tensor):
    """[B, T, heads, head_dim] whose tokens may lie further apart than they are long (a part of a fused projection):
    the struct and the distance in elements."""
    b, n, h, d = t.shape
    pitch = t.stride(1) if n > 1 else (t.stride(0) if b > 1 else h * d)
    dense_heads = (d == 1 or t.stride(3) == 1) and (h == 1 or t.stride(2) == d)
    if not dense_heads or (b > 1 and n > 1 and t.stride(0) != n * pitch):
        raise ValueError("tokens are [batch, tokens, heads, head_dim] with dense heads and one distance between tokens")
    if b * n > 1 and pitch < h * d:
        # (a broadcast view has a distance of 0, which the library takes for `dense`)
        raise ValueError("tokens overlap: a broadcast or overlapping view has to be made contiguous first")
    return _meta(tuple(t.shape), 3, _DTYPES[t.dtype], t.data_ptr()), pitch


def _append_args(cache: Cache4, k: torch.Tensor, v: torch.Tensor, page_table, lengths):
    _on_gpu(k, v, cache.data, page_table, lengths)
    sk, pk = _tokens_struct(k)
    sv, pv = _tokens_struct(v)
    if pk != pv:
        raise ValueError("k and v have one distance between tokens")
    return (ctypes.byref(_cache4_struct(cache)), ctypes.byref(sk), ctypes.byref(sv), pk,
            ctypes.byref(_pages_struct(page_table, lengths)))


def gl_cache4_append(cache: Cache4, k: torch.Tensor, v: torch.Tensor, page_table: torch.Tensor, lengths: torch.Tensor,
                     stream=None) -> None:
    _check(LIB.gl_cache4_append(*_append_args(cache, k, v, page_table, lengths), _stream(stream)), "gl_cache4_append")


def _read_args(cache: Cache4, k: torch.Tensor, v: torch.Tensor, page_table, lengths):
    _on_gpu(k, v, cache.data, page_table, lengths)
    return (ctypes.byref(_cache4_struct(cache)), ctypes.byref(_pages_struct(page_table, lengths)),
            ctypes.byref(_struct(AccessPattern(k, 3))), ctypes.byref(_struct(AccessPattern(v, 3))))


def gl_cache4_read(cache: Cache4, tokens: int, page_table: torch.Tensor, lengths: torch.Tensor, stream=None):
    """The values of the last `tokens` tokens of every sequence: (k, v), bf16 [B, tokens, kv_heads, head_dim]."""
    shape = (page_table.shape[0], tokens, cache.kv_heads, cache.head_dim)
    k, v = (_empty(shape, torch.bfloat16, cache.data.device, stream) for _ in range(2))
    _check(LIB.gl_cache4_read(*_read_args(cache, k, v, page_table, lengths), _stream(stream)), "gl_cache4_read")
    return k, v


def gl_attend_cache4_workspace(q: AccessPattern, cache: Cache4) -> int:
    return int(LIB.gl_attend_cache4_workspace(ctypes.byref(_tokens_struct(q.tensor)[0]), ctypes.byref(_cache4_struct(cache))))


def _attend_args(q, cache, page_table, lengths, out, scale, flags, workspace):
    _on_gpu(q.tensor, cache.data, page_table, lengths, out.tensor, workspace)
    sq, pitch = _tokens_struct(q.tensor)
    sq.access_ndim = q.access_ndim
    return (ctypes.byref(sq), pitch, ctypes.byref(_cache4_struct(cache)), ctypes.byref(_pages_struct(page_table, lengths)),
            float(scale), ctypes.byref(_struct(out)), flags, *_ws(workspace))


def gl_attend_cache4(q: AccessPattern, cache: Cache4, page_table: torch.Tensor, lengths: torch.Tensor,
                     scale: Optional[float] = None, out: Optional[AccessPattern] = None, flags: int = 0,
                     workspace: Optional[torch.Tensor] = None, stream=None) -> AccessPattern:
    """q ((B, T, heads),(head_dim)); scale defaults to 1 / sqrt(head_dim)."""
    if scale is None:
        scale = cache.head_dim ** -0.5
    if out is None:
        dtype = torch.bfloat16 if flags & GL_OUT_BF16 else torch.float32
        out = AccessPattern(_empty(tuple(q.tensor.shape), dtype, q.tensor.device, stream), 3)
    if workspace is None:
        workspace = _scratch(gl_attend_cache4_workspace(q, cache), q.tensor.device, stream)
    _check(LIB.gl_attend_cache4(*_attend_args(q, cache, page_table, lengths, out, scale, flags, workspace), _stream(stream)),
           "gl_attend_cache4")
    return out


def gl_poll_device_status(stream=None) -> int:
    return int(LIB.gl_poll_device_status(_stream(stream)))


def gl_selftest_bounded_wait(limit_ms: int, stream=None) -> None:
    _check(LIB.gl_selftest_bounded_wait(limit_ms, _stream(stream)), "gl_selftest_bounded_wait")


def gl_strerror(code: int) -> str:
    return LIB.gl_strerror(code).decode()


def gl_version() -> int:
    return int(LIB.gl_version())


def _converted(fn, args):
    """`fn` without argument types and `args` as the C values that its types make of them: ctypes otherwise converts every one of
    them on every call (0.5 us of 0.9)."""
    types = getattr(fn, "argtypes", None)
    if types is None:
        return fn, args
    bare = _BARE[fn.__name__]
    values = []
    for value, kind in zip(args, types):
        if issubclass(kind, ctypes._Pointer):
            value, kind = ctypes.addressof(value._obj) if value is not None else None, ctypes.c_void_p
        values.append(kind(value))
    return bare, tuple(values)


class Prepared:
    """A device call with its argument structures built once, for launch loops
    where Python marshalling would otherwise outweigh a microsecond-scale kernel.
    The stream is looked up at call time, so a prepared call can be captured
    into a CUDA graph.  `scratch`: a workspace that nobody else holds.  It was taken
    on the stream that was current then, so torch is told of every other stream
    that uses it: dropping the call then waits for them.  `gpu`: the index of the
    GPU that has to be current."""

    def __init__(self, fn, args, keep, scratch=None, gpu=None):
        self._fn, self._args, self._keep, self._scratch, self._gpu = fn, args, keep, scratch, gpu
        self._streams = None if scratch is None else {_stream(None)}
        if gpu is not None:
            self._keep = (keep, args)                      # (the structures behind the addresses)
            self._fn, self._args = _converted(fn, args)
            self._raw = None, None

    def _on_gpu_call(self, stream):
        if torch._C._cuda_getDevice() != self._gpu:
            _current_is(self._gpu)
        raw = torch._C._cuda_getCurrentRawStream(self._gpu) if stream is None else _stream(stream)
        last = self._raw            # (read once: another thread may put its own stream there at any time)
        if raw != last[0]:
            last = self._raw = raw, ctypes.c_void_p(raw)
        return last

    def __call__(self, stream=None):
        if self._gpu is not None:
            raw, last = self._on_gpu_call(stream)
        else:
            raw = last = _stream(stream)
        if self._streams is not None and raw not in self._streams:
            self._scratch.record_stream(_stream_object(torch.cuda.current_stream() if stream is None else stream))
            self._streams.add(raw)
        rc = self._fn(*self._args, last)
        if rc != GL_OK:
            raise GlError(rc, self._fn.__name__)


def _ws(workspace):
    if workspace is None:
        return 0, 0
    ptr = (workspace.data_ptr() + 1023) // 1024 * 1024
    return ptr, workspace.numel() * workspace.element_size() - (ptr - workspace.data_ptr())


def prepare_cartesian_dot(a0: AccessPattern, w: Optional[GlWindows], a1: AccessPattern, out: AccessPattern,
                          flags: int = 0, workspace: Optional[torch.Tensor] = None) -> Prepared:
    s0, s1, so = _struct(a0), _struct(a1), _struct(out)
    ws_ptr, ws_bytes = _ws(workspace)
    args = (ctypes.byref(s0), _wptr(w), ctypes.byref(s1), ctypes.byref(so), flags, ws_ptr, ws_bytes)
    return Prepared(LIB.gl_cartesian_dot, args, (s0, s1, so, w, a0, a1, out, workspace))


def prepare_access_windows(a: AccessPattern, w: GlWindows, out: AccessPattern) -> Prepared:
    sa, so = _struct(a), _struct(out)
    return Prepared(LIB.gl_access_windows, (ctypes.byref(sa), ctypes.byref(w), ctypes.byref(so)), (sa, so, w, a, out))


def prepare_access_transpose(a: AccessPattern, perm, out: AccessPattern) -> Prepared:
    sa, so = _struct(a), _struct(out)
    arr = (ctypes.c_int32 * len(perm))(*perm)
    return Prepared(LIB.gl_access_transpose, (ctypes.byref(sa), arr, ctypes.byref(so)), (sa, so, arr, a, out))


def prepare_compute_reduce_max(a: AccessPattern, w: Optional[GlWindows], out: AccessPattern) -> Prepared:
    sa, so = _struct(a), _struct(out)
    return Prepared(LIB.gl_compute_reduce_max, (ctypes.byref(sa), _wptr(w), ctypes.byref(so)), (sa, so, w, a, out))


def prepare_access_pad(a: AccessPattern, dim: int, lo: int, hi: int, pad_kind: int, out: AccessPattern) -> Prepared:
    sa, so = _struct(a), _struct(out)
    return Prepared(LIB.gl_access_pad, (ctypes.byref(sa), dim, lo, hi, pad_kind, ctypes.byref(so)), (sa, so, a, out))


def prepare_compute_relu(a: AccessPattern, out: AccessPattern) -> Prepared:
    sa, so = _struct(a), _struct(out)
    return Prepared(LIB.gl_compute_relu, (ctypes.byref(sa), ctypes.byref(so)), (sa, so, a, out))


def prepare_mx4_quantize(a: AccessPattern, out: Mx4) -> Prepared:
    _on_gpu(a.tensor, out.data, out.scale)
    return Prepared(LIB.gl_mx4_quantize, (ctypes.byref(_struct(a)), ctypes.byref(_mx4_struct(out))), (a, out))


def prepare_mx4_dequantize(m: Mx4, out: AccessPattern) -> Prepared:
    _on_gpu(m.data, m.scale, out.tensor)
    return Prepared(LIB.gl_mx4_dequantize, (ctypes.byref(_mx4_struct(m)), ctypes.byref(_struct(out))), (m, out))


def prepare_cartesian_dot_mx4(a0: Mx4, a1: Mx4, out: AccessPattern, flags: int = 0) -> Prepared:
    _on_gpu(a0.data, a0.scale, a1.data, a1.scale, out.tensor)
    return Prepared(LIB.gl_cartesian_dot_mx4, (ctypes.byref(_mx4_struct(a0)), ctypes.byref(_mx4_struct(a1)),
                                               ctypes.byref(_struct(out)), flags), (a0, a1, out))


def prepare_dense_mx4(a0: AccessPattern, a1: Mx4, out: AccessPattern, flags: int = 0,
                      workspace: Optional[torch.Tensor] = None) -> Prepared:
    scratch = None if workspace is not None else _scratch(gl_dense_mx4_workspace(a0, a1), a0.tensor.device)
    workspace = scratch if workspace is None else workspace
    _on_gpu(a0.tensor, a1.data, a1.scale, out.tensor, workspace)
    return Prepared(LIB.gl_dense_mx4, (ctypes.byref(_struct(a0)), ctypes.byref(_mx4_struct(a1)), ctypes.byref(_struct(out)), flags,
                                       *_ws(workspace)), (a0, a1, out, workspace), scratch)


def prepare_f8_quantize(a: AccessPattern, out: F8) -> Prepared:
    gpu = _on_this_gpu(a.tensor, out.data, out.scale)
    return Prepared(LIB.gl_f8_quantize, (ctypes.byref(_struct(a)), ctypes.byref(_f8_struct(out))), (a, out), gpu=gpu)


def prepare_f8_dequantize(m: F8, out: AccessPattern) -> Prepared:
    gpu = _on_this_gpu(m.data, m.scale, out.tensor)
    return Prepared(LIB.gl_f8_dequantize, (ctypes.byref(_f8_struct(m)), ctypes.byref(_struct(out))), (m, out), gpu=gpu)


def prepare_cartesian_dot_f8(a0: F8, a1: F8, out: AccessPattern, flags: int = 0) -> Prepared:
    gpu = _on_this_gpu(a0.data, a0.scale, a1.data, a1.scale, out.tensor)
    return Prepared(LIB.gl_cartesian_dot_f8, (ctypes.byref(_f8_struct(a0)), ctypes.byref(_f8_struct(a1)),
                                              ctypes.byref(_struct(out)), flags), (a0, a1, out), gpu=gpu)


def prepare_dense_f8(a0: AccessPattern, a1: F8, out: AccessPattern, flags: int = 0,
                     workspace: Optional[torch.Tensor] = None) -> Prepared:
    gpu = _on_this_gpu(a0.tensor, a1.data, a1.scale, out.tensor, workspace)
    scratch = None if workspace is not None else _scratch(gl_dense_f8_workspace(a0, a1), a0.tensor.device)
    workspace = scratch if workspace is None else workspace
    return Prepared(LIB.gl_dense_f8, (ctypes.byref(_struct(a0)), ctypes.byref(_f8_struct(a1)), ctypes.byref(_struct(out)), flags,
                                      *_ws(workspace)), (a0, a1, out, workspace), scratch, gpu)


def prepare_compute_norm_rms(x: AccessPattern, weight: Optional[AccessPattern], out, eps: float = 1e-6,
                             residual: Optional[AccessPattern] = None, total: Optional[AccessPattern] = None) -> Prepared:
    """out: an access pattern or an F8 operand."""
    call, args = _norm_call(x, weight, out, eps, residual, total)
    return Prepared(call, args, (x, weight, out, residual, total), gpu=x.tensor.device.index)


def prepare_compute_rotate(x: AccessPattern, plan: GlRotary, positions: torch.Tensor, out: AccessPattern, flags: int = 0) -> Prepared:
    args = _rotate_args(x, plan, positions, out, flags)
    return Prepared(LIB.gl_compute_rotate, args, (x, plan, positions, out), gpu=x.tensor.device.index)


def prepare_cache4_append(cache: Cache4, k, v, page_table, lengths) -> Prepared:
    return Prepared(LIB.gl_cache4_append, _append_args(cache, k, v, page_table, lengths), (cache, k, v, page_table, lengths))


def prepare_cache4_read(cache: Cache4, k, v, page_table, lengths) -> Prepared:
    return Prepared(LIB.gl_cache4_read, _read_args(cache, k, v, page_table, lengths), (cache, k, v, page_table, lengths))


def prepare_attend_cache4(q: AccessPattern, cache: Cache4, page_table, lengths, out: AccessPattern,
                          scale: Optional[float] = None, flags: int = 0, workspace: Optional[torch.Tensor] = None) -> Prepared:
    scratch = None if workspace is not None else _scratch(gl_attend_cache4_workspace(q, cache), q.tensor.device)
    workspace = scratch if workspace is None else workspace
    args = _attend_args(q, cache, page_table, lengths, out, cache.head_dim ** -0.5 if scale is None else scale, flags, workspace)
    return Prepared(LIB.gl_attend_cache4, args, (q, cache, page_table, lengths, out, workspace), scratch)


def output_like(shape_fn_result, device) -> AccessPattern:
    """Allocate the output described by a gl_shape_* result (shape, access_ndim, dtype)."""
    shape, na, dt = shape_fn_result
    return AccessPattern(torch.empty(shape, dtype=_TORCH[dt], device=device), na)
