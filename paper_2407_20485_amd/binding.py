"""Binding of liba2sf.so - argument marshalling only: through ctypes, and for the plain calls of a serving loop (tensors,
ints, floats, a Cache) through the host extension _call.so, which does the same without the interpreter (all through ctypes, with
a warning, where it is missing or was built for another torch).

Every function has the name and the arguments of its C entry point (include/a2sf.h).
torch tensors are accepted wherever the C side takes a device pointer; torch is used for
device memory and for the current stream handle, nothing else.  There is no CPU fallback:
if the shared library is missing the import of a symbol fails loudly.
"""
from __future__ import annotations

import ctypes
import os
import sys
import warnings

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liba2sf.so")

A2SF_OK, A2SF_EINVAL, A2SF_ESHAPE, A2SF_EDTYPE, A2SF_ECAPACITY, A2SF_EWORKSPACE, A2SF_EHIP = range(7)
A2SF_F32, A2SF_BF16, A2SF_E4M3 = 0, 1, 2
A2SF_EVICT_FAST, A2SF_EVICT_STABLE = 0, 1
A2SF_MAX_CAPACITY = 36864
A2SF_STATIC_WS_BYTES = 16 << 20
A2SF_MAX_ROW, A2SF_MAX_VOCABULARY, A2SF_MAX_ROTARY_PARTS = 65536, 4194304, 4
A2SF_WIDE_SUMS = 0x100
A2SF_NO_WINDOW, A2SF_MAX_ALTERNATIVES = 0x7FFFFFFF, 64

EXPORTS = ("a2sf_workspace_bytes", "a2sf_prefill", "a2sf_decode_step", "a2sf_select",
           "a2sf_compact", "a2sf_status_string", "a2sf_prefill_alpha_per_head",
           "a2sf_decode_step_alpha_per_head", "a2sf_ideal_similarity", "a2sf_decode_step_static_ws",
           "a2sf_similarity_mean", "a2sf_decode_plan", "a2sf_prefill_windowed",
           "a2sf_prefill_chunk", "a2sf_prefill_gqa", "a2sf_decode_step_gqa", "a2sf_prefill_chunk_gqa",
           "a2sf_rms_norm", "a2sf_quantize", "a2sf_quantize_weight", "a2sf_matmul_workspace_bytes", "a2sf_matmul_scaled",
           "a2sf_rotary", "a2sf_rotary_table", "a2sf_sample",
           "a2sf_paged_append", "a2sf_paged_attention", "a2sf_paged_workspace_bytes", "a2sf_log_probs")


class Budget(ctypes.Structure):
    _fields_ = [("select", ctypes.c_int32), ("recent", ctypes.c_int32)]


class CacheStruct(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("scores", ctypes.c_void_p),
                ("pos", ctypes.c_void_p), ("len", ctypes.c_void_p), ("G", ctypes.c_int32),
                ("capacity", ctypes.c_int32), ("d", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("stride", ctypes.c_int64)]


class Rows8(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("stride", ctypes.c_int64),
                ("scale_stride", ctypes.c_int64)]


class RotaryPart(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("y", ctypes.c_void_p), ("x_stride", ctypes.c_int64 * 3),
                ("y_stride", ctypes.c_int64 * 3), ("heads", ctypes.c_int32), ("rotate", ctypes.c_int32)]


class PagesStruct(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scales", ctypes.c_void_p), ("v_scales", ctypes.c_void_p),
                ("stride", ctypes.c_int64 * 3), ("scale_stride", ctypes.c_int64 * 3), ("pages", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("d", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class Sequences(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("len", ctypes.c_void_p), ("starts", ctypes.c_void_p), ("table_stride", ctypes.c_int64),
                ("sequences", ctypes.c_int32), ("table_pages", ctypes.c_int32)]


class Heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("stride", ctypes.c_int64 * 2)]


_lib = None
_call = None  # the extension, loaded with the library


def lib() -> ctypes.CDLL:
    """The loaded shared library; raises if it has not been built."""
    global _lib, _call
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2407_20485_amd.build` "
                "(there is no fallback path)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, f32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_float, ctypes.c_size_t
        L.a2sf_workspace_bytes.restype = sz
        L.a2sf_workspace_bytes.argtypes = [i32, i32, i32, i32, i32, Budget]
        L.a2sf_prefill.restype = i32
        L.a2sf_prefill.argtypes = [vp, vp, vp, i32, f32, Budget, ctypes.POINTER(CacheStruct), vp, vp,
                                   vp, sz, vp]
        L.a2sf_prefill_windowed.restype = i32
        L.a2sf_prefill_windowed.argtypes = [vp, vp, vp, i32, f32, f32, Budget, ctypes.POINTER(CacheStruct), vp,
                                            vp, vp, sz, vp]
        L.a2sf_prefill_chunk.restype = i32
        L.a2sf_prefill_chunk.argtypes = [vp, vp, vp, i32, i32, f32, Budget, ctypes.POINTER(CacheStruct), vp,
                                         vp, sz, vp]
        L.a2sf_prefill_chunk_gqa.restype = i32
        L.a2sf_prefill_chunk_gqa.argtypes = [vp, vp, vp, i32, i32, i32, f32, Budget, ctypes.POINTER(CacheStruct),
                                             vp, vp, sz, vp]
        L.a2sf_prefill_gqa.restype = i32
        L.a2sf_prefill_gqa.argtypes = [vp, vp, vp, i32, i32, f32, Budget, ctypes.POINTER(CacheStruct), vp, vp,
                                       vp, sz, vp]
        L.a2sf_decode_step_gqa.restype = i32
        L.a2sf_decode_step_gqa.argtypes = [vp, vp, vp, i32, ctypes.POINTER(CacheStruct), i32, f32, Budget, i32,
                                           vp, vp, sz, vp]
        L.a2sf_decode_step.restype = i32
        L.a2sf_decode_step.argtypes = [vp, vp, vp, i32, ctypes.POINTER(CacheStruct), f32, Budget, i32,
                                       vp, vp, sz, vp]
        L.a2sf_decode_step_static_ws.restype = i32
        L.a2sf_decode_step_static_ws.argtypes = [vp, vp, vp, i32, ctypes.POINTER(CacheStruct), f32, Budget,
                                                 i32, vp, vp]
        L.a2sf_prefill_alpha_per_head.restype = i32
        L.a2sf_prefill_alpha_per_head.argtypes = [vp, vp, vp, i32, vp, f32, Budget,
                                                  ctypes.POINTER(CacheStruct), vp, vp, vp, sz, vp]
        L.a2sf_decode_step_alpha_per_head.restype = i32
        L.a2sf_decode_step_alpha_per_head.argtypes = [vp, vp, vp, i32, ctypes.POINTER(CacheStruct), vp,
                                                      Budget, i32, vp, vp, sz, vp]
        L.a2sf_select.restype = i32
        L.a2sf_select.argtypes = [vp, vp, vp, i32, i32, i32, Budget, vp, vp, vp]
        L.a2sf_compact.restype = i32
        L.a2sf_compact.argtypes = [ctypes.POINTER(CacheStruct), vp, i32, vp, vp]
        L.a2sf_ideal_similarity.restype = i32
        L.a2sf_ideal_similarity.argtypes = [vp, vp, i32, i32, ctypes.POINTER(CacheStruct), vp, vp]
        L.a2sf_similarity_mean.restype = i32
        L.a2sf_similarity_mean.argtypes = [vp, i32, i32, i32, vp, vp]
        L.a2sf_decode_plan.restype = i32
        L.a2sf_decode_plan.argtypes = [i32, i32, i32, ctypes.POINTER(i32), ctypes.POINTER(i32),
                                       ctypes.POINTER(i32), ctypes.POINTER(i32)]
        f64, rows, rows8 = ctypes.c_double, ctypes.POINTER(Rows), ctypes.POINTER(Rows8)
        L.a2sf_rms_norm.restype = i32
        L.a2sf_rms_norm.argtypes = [rows, rows, vp, f32, i32, i32, i32, rows, rows, rows8, vp]
        L.a2sf_quantize.restype = i32
        L.a2sf_quantize.argtypes = [rows, rows, i32, i32, i32, rows, rows8, vp]
        L.a2sf_quantize_weight.restype = i32
        L.a2sf_quantize_weight.argtypes = [rows, i32, i32, i32, rows8, vp]
        L.a2sf_matmul_workspace_bytes.restype = sz
        L.a2sf_matmul_workspace_bytes.argtypes = [i32, i32, i32]
        L.a2sf_matmul_scaled.restype = i32
        L.a2sf_matmul_scaled.argtypes = [rows8, rows8, i32, i32, i32, rows, i32, vp, sz, vp]
        L.a2sf_rotary.restype = i32
        L.a2sf_rotary.argtypes = [ctypes.POINTER(RotaryPart), i32, i32, i32, i32, i32, vp, ctypes.c_int64, vp, i32, i32,
                                  i32, i32, vp]
        L.a2sf_rotary_table.restype = i32
        L.a2sf_rotary_table.argtypes = [vp, i32, i32, f64, f64, i32, f64, f64, f64, vp]
        L.a2sf_sample.restype = i32
        L.a2sf_sample.argtypes = [rows, rows, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp]
        heads, pages, seqs = ctypes.POINTER(Heads), ctypes.POINTER(PagesStruct), ctypes.POINTER(Sequences)
        L.a2sf_paged_append.restype = i32
        L.a2sf_paged_append.argtypes = [heads, heads, heads, i32, i32, i32, seqs, pages, vp, i32, i32, i32, heads, vp]
        L.a2sf_paged_attention.restype = i32
        L.a2sf_paged_attention.argtypes = [heads, i32, i32, i32, seqs, pages, i32, i32, heads, vp, sz, vp]
        L.a2sf_paged_workspace_bytes.restype = sz
        L.a2sf_paged_workspace_bytes.argtypes = [i32, i32, i32, i32, i32, ctypes.c_int64]
        L.a2sf_log_probs.restype = i32
        L.a2sf_log_probs.argtypes = [rows, i32, i32, i32, rows, i32, rows, vp, rows, rows, i32, vp]
        L.a2sf_status_string.restype = ctypes.c_char_p
        L.a2sf_status_string.argtypes = [i32]
        if _call is None:
            _call = _load_extension()
        L.at = {name: ctypes.cast(getattr(L, name), vp).value for name in EXPORTS}
        _lib = L
    return _lib


class _NoExtension:
    """Every call goes through ctypes."""

    @staticmethod
    def _leave(*args):
        return -1

    decode_step = prefill = prefill_chunk = rms_norm = quantize = matmul_scaled = rotary = sample = _leave
    paged_append = paged_attention = log_probs = _leave


def _load_extension():
    """_call, if it is there and was built against this torch and this Python; the library itself needs neither."""
    try:
        from . import _call as extension
        running = f"torch {torch.__version__.split('+')[0]}, Python {sys.version_info[0]}.{sys.version_info[1]}"
        built_for = getattr(extension, "built_for", "something older")
        if built_for != running:
            raise ImportError(f"built for {built_for}, not {running}")
    except ImportError as e:
        warnings.warn(f"{os.path.join(_HERE, '_call.so')} is missing or does not load ({e}): steps, prompts and chunks take 2 us more host "
                      "time each; build it with `python -m paper_2407_20485_amd.build`", RuntimeWarning, stacklevel=3)
        return _NoExtension
    extension.init(Cache, torch.float32, torch.bfloat16, _raw_stream if _get_device else None, _get_device, Pages)
    return extension


class A2SFError(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        super().__init__(f"a2sf status {status}: {a2sf_status_string(status)}")


# The generation step of a few heads takes 7 us on the GPU: the marshalling is on its critical path.  _call takes the calls
# whose arguments are plain and answers -1, having done nothing, to all others; those go through the ctypes form below.
_Tensor = torch.Tensor
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # (absent in builds without a GPU backend)
_get_device = getattr(torch._C, "_cuda_getDevice", None)


def _ptr(x):
    if type(x) is _Tensor or isinstance(x, _Tensor):
        return x.data_ptr()
    return None if x is None else int(x)


def _stream(stream):
    if stream is not None:
        return int(stream)
    if _raw_stream is not None and torch.cuda.is_initialized():
        return _raw_stream(_get_device())
    return torch.cuda.current_stream().cuda_stream if torch.cuda.is_available() else None


def _entry(name: str) -> int:
    return (_lib or lib()).at[name]


def _check(status: int):
    if status != A2SF_OK:
        raise A2SFError(status)


_DTYPE_CODES = {torch.float32: A2SF_F32, torch.bfloat16: A2SF_BF16}


_PAGE_CODES = {**_DTYPE_CODES, torch.float8_e4m3fn: A2SF_E4M3}


def dtype_code(t: torch.dtype) -> int:
    code = _DTYPE_CODES.get(t)
    if code is None:
        raise A2SFError(A2SF_EDTYPE)
    return code


class Cache:
    """Device buffers of a KV cache for G heads plus the matching C struct."""

    def __init__(self, G: int, capacity: int, d: int, dtype: torch.dtype, device="cuda"):
        self.G, self.capacity, self.d, self.dtype = G, capacity, d, dtype
        self.k = torch.zeros((G, capacity, d), dtype=dtype, device=device)
        self.v = torch.zeros((G, capacity, d), dtype=dtype, device=device)
        self.scores = torch.zeros((G, capacity), dtype=torch.float32, device=device)
        self.pos = torch.zeros((G, capacity), dtype=torch.int32, device=device)
        self.len = torch.zeros((G,), dtype=torch.int32, device=device)

    def struct(self) -> CacheStruct:
        return CacheStruct(self.k.data_ptr(), self.v.data_ptr(), self.scores.data_ptr(),
                           self.pos.data_ptr(), self.len.data_ptr(), self.G, self.capacity, self.d,
                           dtype_code(self.dtype))

    def tensors(self):
        return (self.k, self.v, self.scores, self.pos, self.len)

    def snapshot(self):
        return [t.clone() for t in self.tensors()]

    def restore(self, snap):
        for t, s in zip(self.tensors(), snap):
            t.copy_(s)


class Pages:
    """Device buffers of a paged KV cache: k, v [pages, kv_heads, page_size, d], and for 8 bits (torch.float8_e4m3fn) the bytes of
    their scales [pages, kv_heads, page_size]; with the matching C struct, made once, so the tensors stay the ones they are."""

    def __init__(self, pages: int, page_size: int, kv_heads: int, d: int, dtype: torch.dtype, device="cuda"):
        shape, eight = (pages, kv_heads, page_size, d), dtype == torch.float8_e4m3fn
        k, v = (torch.zeros(shape, dtype=dtype, device=device) for _ in range(2))
        ks, vs = (torch.zeros(shape[:3], dtype=torch.uint8, device=device) if eight else None for _ in range(2))
        self._take(k, v, ks, vs)

    @classmethod
    def of(cls, k, v, k_scales=None, v_scales=None) -> "Pages":
        """Pages in tensors that are there already: views of any strides with a row's elements next to each other, k and v alike."""
        self = cls.__new__(cls)
        self._take(k, v, k_scales, v_scales)
        return self

    def _take(self, k, v, k_scales, v_scales):
        _need(k.dim() == 4 and v.shape == k.shape and v.stride() == k.stride() and k.stride(3) == 1)
        _need(k.dtype in _PAGE_CODES and v.dtype == k.dtype, A2SF_EDTYPE)
        _need((k.dtype == torch.float8_e4m3fn) == (k_scales is not None) == (v_scales is not None), A2SF_EINVAL)
        _reach(v, k)
        scale_stride = (0, 0, 0)
        if k_scales is not None:
            _need(k_scales.shape == k.shape[:3] and v_scales.shape == k.shape[:3] and k_scales.stride() == v_scales.stride())
            _need(k_scales.dtype == torch.uint8 and v_scales.dtype == torch.uint8, A2SF_EDTYPE)
            _reach(k_scales, k)
            _reach(v_scales, k)
            scale_stride = k_scales.stride()
        self.k, self.v, self.k_scales, self.v_scales = k, v, k_scales, v_scales
        self.pages, self.kv_heads, self.page_size, self.d = k.shape
        _int32(*k.shape)
        self.dtype = k.dtype
        three = ctypes.c_int64 * 3
        self.struct = PagesStruct(k.data_ptr(), v.data_ptr(), _ptr(k_scales), _ptr(v_scales), three(*k.stride()[:3]), three(*scale_stride),
                                  self.pages, self.page_size, self.kv_heads, self.d, _PAGE_CODES[k.dtype])
        self.address = ctypes.addressof(self.struct)

    def tensors(self):
        return tuple(t for t in (self.k, self.v, self.k_scales, self.v_scales) if t is not None)


def _cache_struct(cache):
    return cache.struct() if isinstance(cache, Cache) else cache


def a2sf_status_string(status: int) -> str:
    return lib().a2sf_status_string(int(status)).decode()


def a2sf_workspace_bytes(G, n_max, capacity, d, dtype, select, recent) -> int:
    return int(lib().a2sf_workspace_bytes(G, n_max, capacity, d, dtype, Budget(select, recent)))


def a2sf_prefill(q, k, v, n, alpha, select, recent, cache, o=None, scores_full=None,
                 workspace=None, workspace_bytes=None, stream=None):
    at = _entry("a2sf_prefill")
    status = _call.prefill(at, q, k, v, n, None, alpha, select, recent, cache, o, scores_full, workspace,
                           workspace_bytes, stream)
    if status >= 0:
        return _check(status)
    cs = _cache_struct(cache)
    if workspace_bytes is None:
        workspace_bytes = workspace.nbytes if workspace is not None else 0
    _check(lib().a2sf_prefill(_ptr(q), _ptr(k), _ptr(v), n, alpha, Budget(select, recent),
                              ctypes.byref(cs), _ptr(o), _ptr(scores_full), _ptr(workspace),
                              workspace_bytes, _stream(stream)))


def a2sf_prefill_windowed(q, k, v, n, alpha, score_rel_tol, select, recent, cache, o=None, scores_full=None,
                          workspace=None, workspace_bytes=None, stream=None):
    cs = _cache_struct(cache)
    if workspace_bytes is None:
        workspace_bytes = workspace.nbytes if workspace is not None else 0
    _check(lib().a2sf_prefill_windowed(_ptr(q), _ptr(k), _ptr(v), n, alpha, score_rel_tol,
                                       Budget(select, recent), ctypes.byref(cs), _ptr(o), _ptr(scores_full),
                                       _ptr(workspace), workspace_bytes, _stream(stream)))


def a2sf_prefill_chunk(q, k, v, m, pos0, alpha, select, recent, cache, o=None, workspace=None,
                       workspace_bytes=None, stream=None):
    at = _entry("a2sf_prefill_chunk")
    status = _call.prefill_chunk(at, q, k, v, m, pos0, None, alpha, select, recent, cache, o,
                                 workspace, workspace_bytes, stream)
    if status >= 0:
        return _check(status)
    cs = _cache_struct(cache)
    if workspace_bytes is None:
        workspace_bytes = workspace.nbytes if workspace is not None else 0
    _check(lib().a2sf_prefill_chunk(_ptr(q), _ptr(k), _ptr(v), m, pos0, alpha, Budget(select, recent),
                                    ctypes.byref(cs), _ptr(o), _ptr(workspace), workspace_bytes,
                                    _stream(stream)))


def a2sf_prefill_chunk_gqa(q, k, v, m, pos0, group, alpha, select, recent, cache, o=None, workspace=None,
                           workspace_bytes=None, stream=None):
    at = _entry("a2sf_prefill_chunk_gqa")
    status = _call.prefill_chunk(at, q, k, v, m, pos0, group, alpha, select, recent, cache, o,
                                 workspace, workspace_bytes, stream)
    if status >= 0:
        return _check(status)
    cs = _cache_struct(cache)
    if workspace_bytes is None:
        workspace_bytes = workspace.nbytes if workspace is not None else 0
    _check(lib().a2sf_prefill_chunk_gqa(_ptr(q), _ptr(k), _ptr(v), m, pos0, group, alpha, Budget(select, recent),
                                        ctypes.byref(cs), _ptr(o), _ptr(workspace), workspace_bytes,
                                        _stream(stream)))


def a2sf_prefill_gqa(q, k, v, n, group, alpha, select, recent, cache, o=None, scores_full=None,
                     workspace=None, workspace_bytes=None, stream=None):
    at = _entry("a2sf_prefill_gqa")
    status = _call.prefill(at, q, k, v, n, group, alpha, select, recent, cache, o, scores_full,
                           workspace, workspace_bytes, stream)
    if status >= 0:
        return _check(status)
    cs = _cache_struct(cache)
    if workspace_bytes is None:
        workspace_bytes = workspace.nbytes if workspace is not None else 0
    _check(lib().a2sf_prefill_gqa(_ptr(q), _ptr(k), _ptr(v), n, group, alpha, Budget(select, recent),
                                  ctypes.byref(cs), _ptr(o), _ptr(scores_full), _ptr(workspace),
                                  workspace_bytes, _stream(stream)))


def a2sf_decode_step_gqa(q, k_new, v_new, t_pos, cache, group, alpha, select, recent, o,
                         mode=A2SF_EVICT_FAST, workspace=None, workspace_bytes=None, stream=None):
    at = _entry("a2sf_decode_step_gqa")
    status = _call.decode_step(at, q, k_new, v_new, t_pos, cache, group, alpha, select, recent, o,
                               mode, workspace, workspace_bytes, stream)
    if status >= 0:
        return _check(status)
    cs = _cache_struct(cache)
    if workspace_bytes is None:
        workspace_bytes = workspace.nbytes if workspace is not None else 0
    _check(lib().a2sf_decode_step_gqa(_ptr(q), _ptr(k_new), _ptr(v_new), t_pos, ctypes.byref(cs), group,
                                      alpha, Budget(select, recent), mode, _ptr(o), _ptr(workspace),
                                      workspace_bytes, _stream(stream)))


def a2sf_decode_step(q, k_new, v_new, t_pos, cache, alpha, select, recent, o,
                     mode=A2SF_EVICT_FAST, workspace=None, workspace_bytes=None, stream=None):
    at = _entry("a2sf_decode_step")
    status = _call.decode_step(at, q, k_new, v_new, t_pos, cache, None, alpha, select, recent, o, mode,
                               workspace, workspace_bytes, stream)
    if status >= 0:
        return _check(status)
    cs = _cache_struct(cache)
    if workspace_bytes is None:
        workspace_bytes = workspace.nbytes if workspace is not None else 0
    _check(lib().a2sf_decode_step(_ptr(q), _ptr(k_new), _ptr(v_new), t_pos, ctypes.byref(cs), alpha,
                                  Budget(select, recent), mode, _ptr(o), _ptr(workspace),
                                  workspace_bytes, _stream(stream)))


def a2sf_decode_step_static_ws(q, k_new, v_new, t_pos, cache, alpha, select, recent, o,
                               mode=A2SF_EVICT_FAST, stream=None):
    cs = _cache_struct(cache)
    _check(lib().a2sf_decode_step_static_ws(_ptr(q), _ptr(k_new), _ptr(v_new), t_pos, ctypes.byref(cs),
                                            alpha, Budget(select, recent), mode, _ptr(o), _stream(stream)))


def a2sf_prefill_alpha_per_head(q, k, v, n, alpha_heads, alpha_max, select, recent, cache, o=None,
                                scores_full=None, workspace=None, workspace_bytes=None, stream=None):
    cs = _cache_struct(cache)
    if workspace_bytes is None:
        workspace_bytes = workspace.nbytes if workspace is not None else 0
    _check(lib().a2sf_prefill_alpha_per_head(_ptr(q), _ptr(k), _ptr(v), n, _ptr(alpha_heads), alpha_max,
                                             Budget(select, recent), ctypes.byref(cs), _ptr(o),
                                             _ptr(scores_full), _ptr(workspace), workspace_bytes,
                                             _stream(stream)))


def a2sf_decode_step_alpha_per_head(q, k_new, v_new, t_pos, cache, alpha_heads, select, recent, o,
                                    mode=A2SF_EVICT_FAST, workspace=None, workspace_bytes=None,
                                    stream=None):
    cs = _cache_struct(cache)
    if workspace_bytes is None:
        workspace_bytes = workspace.nbytes if workspace is not None else 0
    _check(lib().a2sf_decode_step_alpha_per_head(_ptr(q), _ptr(k_new), _ptr(v_new), t_pos,
                                                 ctypes.byref(cs), _ptr(alpha_heads),
                                                 Budget(select, recent), mode, _ptr(o), _ptr(workspace),
                                                 workspace_bytes, _stream(stream)))


def a2sf_select(scores, pos, length, G, L, stride, select, recent, keep_idx, n_keep, stream=None):
    _check(lib().a2sf_select(_ptr(scores), _ptr(pos), _ptr(length), G, L, stride,
                             Budget(select, recent), _ptr(keep_idx), _ptr(n_keep), _stream(stream)))


def a2sf_ideal_similarity(q, k_all, n_stride, t_pos, cache, cos_out, stream=None):
    cs = _cache_struct(cache)
    _check(lib().a2sf_ideal_similarity(_ptr(q), _ptr(k_all), n_stride, t_pos, ctypes.byref(cs),
                                       _ptr(cos_out), _stream(stream)))


def a2sf_similarity_mean(cos, steps, G, first_step, mean_out, stream=None):
    _check(lib().a2sf_similarity_mean(_ptr(cos), steps, G, first_step, _ptr(mean_out), _stream(stream)))


def a2sf_decode_plan(G, capacity, d):
    """(nsplit, rows_per_split, wave_slots, wave_heads) of a2sf_decode_step for these sizes."""
    a, b, c, h = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
    _check(lib().a2sf_decode_plan(G, capacity, d, ctypes.byref(a), ctypes.byref(b), ctypes.byref(c),
                                  ctypes.byref(h)))
    return a.value, b.value, c.value, h.value


def a2sf_compact(cache, keep_idx, keep_stride, n_keep, stream=None):
    cs = _cache_struct(cache)
    _check(lib().a2sf_compact(ctypes.byref(cs), _ptr(keep_idx), keep_stride, _ptr(n_keep),
                              _stream(stream)))


# ---- the operators around the attention: rows are 2-D tensors whose sizes, strides and type the C arguments are taken from ----

_EIGHT_BIT = (torch.float8_e4m3fn, torch.uint8)


def _need(ok, status=A2SF_ESHAPE):
    if not ok:
        raise A2SFError(status)


def _int32(*sizes):
    """The C arguments are of 32 bits, and ctypes would cut larger ones off."""
    _need(max(sizes) <= 0x7FFFFFFF)


def _reach(x, like):
    """x is memory that the GPU of `like` can read: its own, or pinned memory of the host."""
    if x.device != like.device:
        _need(not like.is_cuda if x.is_cuda else x.device.type == "cpu" and x.is_pinned(), A2SF_EINVAL)


def _stream_of(first, stream):
    """The stream of a call that takes its sizes from `first`, which has to be such memory too."""
    _need(first.is_cuda or not torch.cuda.is_available() or first.is_pinned(), A2SF_EINVAL)
    return _stream(stream)


def _rows(x, like, dtype=None):
    """The C struct of [rows, n] (None of None); `like`: the tensor whose sizes (and type, unless one is named) it has to have."""
    if x is None:
        return None
    _reach(x, like)
    _need(x.dim() == 2 and x.shape == like.shape and (x.stride(1) == 1 or x.shape[1] == 1))
    _need(x.dtype == (dtype or like.dtype), A2SF_EDTYPE)
    return Rows(x.data_ptr(), x.stride(0))


def _rows8(q, scales, rows, n, like, scale_rows=None):
    """... of 8-bit rows [rows, n] (torch.float8_e4m3fn, or uint8 for their bytes) and scales [scale_rows, ceil(n / 128)] uint8."""
    if q is None and scales is None:
        return None
    _need(q is not None and scales is not None, A2SF_EINVAL)
    _reach(q, like)
    _reach(scales, like)
    _need(q.dtype in _EIGHT_BIT and scales.dtype == torch.uint8, A2SF_EDTYPE)
    _need(tuple(q.shape) == (rows, n) and (q.stride(1) == 1 or n == 1))
    _need(tuple(scales.shape) == (scale_rows or rows, -(-n // 128)) and (scales.stride(1) == 1 or n <= 128))
    return Rows8(q.data_ptr(), scales.data_ptr(), q.stride(0), scales.stride(0))


def _column(x, rows, dtype, like):
    """The address of [rows] (None of None)."""
    if x is None:
        return None
    _reach(x, like)
    _need(x.dim() == 1 and x.shape[0] == rows and (x.stride(0) == 1 or rows == 1))
    _need(x.dtype == dtype, A2SF_EDTYPE)
    return x.data_ptr()


def a2sf_rms_norm(x, weight, eps, residual=None, total=None, out=None, q=None, scales=None, stream=None):
    at = _entry("a2sf_rms_norm")
    status = _call.rms_norm(at, x, weight, eps, residual, total, out, q, scales, stream)
    if status >= 0:
        return _check(status)
    _need(x.dim() == 2)
    rows, n = x.shape
    _int32(rows, n)
    _check(lib().a2sf_rms_norm(_rows(x, x), _rows(residual, x), _column(weight, n, x.dtype, x), eps, rows, n, dtype_code(x.dtype),
                               _rows(total, x), _rows(out, x), _rows8(q, scales, rows, n, x), _stream_of(x, stream)))


def a2sf_quantize(x, q, scales, gate=None, out=None, stream=None):
    at = _entry("a2sf_quantize")
    status = _call.quantize(at, x, q, scales, gate, out, stream)
    if status >= 0:
        return _check(status)
    _need(x.dim() == 2)
    rows, n = x.shape
    _int32(rows, n)
    _check(lib().a2sf_quantize(_rows(x, x), _rows(gate, x), rows, n, dtype_code(x.dtype), _rows(out, x),
                               _rows8(q, scales, rows, n, x), _stream_of(x, stream)))


def a2sf_quantize_weight(w, q, scales, stream=None):
    _need(w.dim() == 2)
    n, k = w.shape
    _int32(n, k)
    _check(lib().a2sf_quantize_weight(_rows(w, w), n, k, dtype_code(w.dtype), _rows8(q, scales, n, k, w, -(-n // 128)),
                                      _stream_of(w, stream)))


def a2sf_matmul_workspace_bytes(m, n, k) -> int:
    return int(lib().a2sf_matmul_workspace_bytes(m, n, k)) if max(m, n, k) <= 0x7FFFFFFF else 0


def a2sf_matmul_scaled(a, a_scales, b, b_scales, c, workspace=None, workspace_bytes=None, stream=None, wide_sums=False):
    """wide_sums: a bfloat16 c too is summed in 32 bits (A2SF_WIDE_SUMS)."""
    at = _entry("a2sf_matmul_scaled")
    status = _call.matmul_scaled(at, a, a_scales, b, b_scales, c, workspace, workspace_bytes, stream, wide_sums)
    if status >= 0:
        return _check(status)
    _need(a.dim() == 2 and b.dim() == 2 and c.dim() == 2)
    m, k = a.shape
    n = b.shape[0]
    _need(tuple(c.shape) == (m, n))
    _int32(m, n, k)
    if workspace_bytes is None:
        workspace_bytes = workspace.nbytes if workspace is not None else 0
    if isinstance(workspace, torch.Tensor):
        _reach(workspace, c)
    _check(lib().a2sf_matmul_scaled(_rows8(a, a_scales, m, k, c), _rows8(b, b_scales, n, k, c, -(-n // 128)), m, n, k, _rows(c, c),
                                    dtype_code(c.dtype) | (A2SF_WIDE_SUMS if wide_sums else 0), _ptr(workspace), workspace_bytes,
                                    _stream_of(c, stream)))


def a2sf_rotary(parts, pos, table, interleaved=False, inverse=False, stream=None):
    """parts: (x, y) or (x, y, rotate), each [batch, length, heads, d] with a head's elements next to each other;
    pos [batch, length] int32; table [rows, rotary_dims] fp32.  interleaved: A2SF_ROTARY_NEIGHBOURS, else A2SF_ROTARY_HALVES."""
    at = _entry("a2sf_rotary")
    status = _call.rotary(at, parts, pos, table, interleaved, inverse, stream)
    if status >= 0:
        return _check(status)
    _need(1 <= len(parts) <= A2SF_MAX_ROTARY_PARTS, A2SF_EINVAL)
    first = parts[0][0]
    _need(first.dim() == 4)
    batch, length, _, d = first.shape
    made = (RotaryPart * len(parts))()
    for to, (x, y, *rotate) in zip(made, parts):
        _need(x.dim() == 4 and x.shape == y.shape and x.shape[:2] == (batch, length) and x.shape[3] == d)
        _need((x.stride(3) == 1 and y.stride(3) == 1) or d == 1)
        _need(x.dtype == first.dtype and y.dtype == first.dtype, A2SF_EDTYPE)
        _reach(x, first)
        _reach(y, first)
        _int32(*x.shape)
        to.x, to.y, to.heads, to.rotate = x.data_ptr(), y.data_ptr(), x.shape[2], int(rotate[0]) if rotate else 1
        to.x_stride[:], to.y_stride[:] = x.stride()[:3], y.stride()[:3]
    _need(tuple(pos.shape) == (batch, length) and (pos.stride(1) == 1 or length == 1))
    _need(table.dim() == 2 and table.is_contiguous())
    _need(pos.dtype == torch.int32 and table.dtype == torch.float32, A2SF_EDTYPE)
    _reach(pos, first)
    _reach(table, first)
    _need(table.shape[1] <= d)
    _int32(table.shape[0])
    _check(lib().a2sf_rotary(made, len(parts), batch, length, d, dtype_code(first.dtype), pos.data_ptr(), pos.stride(0),
                             table.data_ptr(), table.shape[0], table.shape[1], int(bool(interleaved)), int(bool(inverse)),
                             _stream_of(first, stream)))


def a2sf_rotary_table(table, base=10000.0, factor=1.0, original_length=0, low=0.0, high=0.0, magnitude=1.0, stream=None):
    _need(table.dim() == 2 and table.is_contiguous())
    _need(table.dtype == torch.float32, A2SF_EDTYPE)
    _int32(*table.shape)
    _check(lib().a2sf_rotary_table(table.data_ptr(), table.shape[0], table.shape[1], base, factor, original_length, low,
                                   high, magnitude, _stream_of(table, stream)))


def a2sf_sample(logits, noise, token, temperature=None, top_k=None, top_p=None, min_p=None, prob=None, stream=None):
    at = _entry("a2sf_sample")
    status = _call.sample(at, logits, noise, token, temperature, top_k, top_p, min_p, prob, stream)
    if status >= 0:
        return _check(status)
    _need(logits.dim() == 2)
    rows, n = logits.shape
    _int32(rows, n)
    f = torch.float32
    _check(lib().a2sf_sample(_rows(logits, logits), _rows(noise, logits, f), rows, n, dtype_code(logits.dtype),
                             _column(temperature, rows, f, logits), _column(top_k, rows, torch.int32, logits),
                             _column(top_p, rows, f, logits), _column(min_p, rows, f, logits),
                             _column(token, rows, torch.int32, logits), _column(prob, rows, f, logits),
                             _stream_of(logits, stream)))


# ---- keys and values in pages ----

def _heads(x, like, heads=None):
    """The C struct of [tokens, heads, d]; `like`: the tensor whose tokens, d and type it has to have."""
    _reach(x, like)
    _need(x.dim() == 3 and x.shape[0] == like.shape[0] and x.shape[2] == like.shape[2] and (heads is None or x.shape[1] == heads))
    _need(x.stride(2) == 1 or x.shape[2] == 1)
    _need(x.dtype == like.dtype, A2SF_EDTYPE)
    return Heads(x.data_ptr(), (ctypes.c_int64 * 2)(x.stride(0), x.stride(1)))


def _sequences(table, lens, starts, like):
    """... of table [sequences, table_pages], lens [sequences] and starts [sequences + 1] (or None), all int32."""
    _need(table.dim() == 2 and (table.stride(1) == 1 or table.shape[1] == 1))
    _need(table.dtype == torch.int32, A2SF_EDTYPE)
    _reach(table, like)
    n = table.shape[0]
    _int32(*table.shape)
    return Sequences(table.data_ptr(), _column(lens, n, torch.int32, like), _column(starts, n + 1, torch.int32, like), table.stride(0), n,
                     table.shape[1])


def a2sf_paged_append(q, k, v, cache, table, lens, starts=None, q_out=None, rotary=None, interleaved=False, stream=None):
    """q [tokens, heads, d] (with q_out; both may be None), k, v [tokens, kv_heads, d] into the pages of `cache` (Pages); table, lens and
    starts as in a2sf_sequences; rotary: the table [rows, rotary_dims] of a2sf_rotary_table, None: nothing is turned."""
    at = _entry("a2sf_paged_append")
    status = _call.paged_append(at, q, k, v, cache, table, lens, starts, q_out, rotary, interleaved, stream)
    if status >= 0:
        return _check(status)
    _need(k.dim() == 3 and k.shape[2] == cache.d)
    _need((q is None) == (q_out is None), A2SF_EINVAL)
    _reach(cache.k, k)
    tokens, heads = k.shape[0], 0 if q is None else q.shape[1]
    _int32(tokens, heads)
    rows = dims = 0
    if rotary is not None:
        _need(rotary.dim() == 2 and rotary.is_contiguous())
        _need(rotary.dtype == torch.float32, A2SF_EDTYPE)
        _reach(rotary, k)
        rows, dims = rotary.shape
        _int32(rows, dims)
    _check(lib().a2sf_paged_append(None if q is None else _heads(q, k), _heads(k, k, cache.kv_heads), _heads(v, k, cache.kv_heads), tokens,
                                   heads, dtype_code(k.dtype), _sequences(table, lens, starts, k), ctypes.byref(cache.struct),
                                   _ptr(rotary), rows, dims, int(bool(interleaved)), None if q is None else _heads(q_out, k, heads),
                                   _stream_of(k, stream)))


def a2sf_paged_attention(q, cache, table, lens, o, starts=None, window=None, sinks=0, workspace=None, workspace_bytes=None, stream=None,
                         wide_sums=False):
    """window: tokens that a token sees, itself among them (None: all).  wide_sums: bfloat16 calls with starts hold probabilities to 2^-17 as
    those without do (A2SF_WIDE_SUMS)."""
    at = _entry("a2sf_paged_attention")
    status = _call.paged_attention(at, q, cache, table, lens, o, starts, window, sinks, workspace, workspace_bytes, stream, wide_sums)
    if status >= 0:
        return _check(status)
    _need(q.dim() == 3 and q.shape[2] == cache.d)
    _reach(cache.k, q)
    tokens, heads = q.shape[:2]
    window = A2SF_NO_WINDOW if window is None else window
    _int32(tokens, heads, window, sinks)
    if workspace_bytes is None:
        workspace_bytes = workspace.nbytes if workspace is not None else 0
    if isinstance(workspace, torch.Tensor):
        _reach(workspace, q)
    _check(lib().a2sf_paged_attention(_heads(q, q), tokens, heads, dtype_code(q.dtype) | (A2SF_WIDE_SUMS if wide_sums else 0),
                                      _sequences(table, lens, starts, q), ctypes.byref(cache.struct), window, sinks, _heads(o, q, heads),
                                      _ptr(workspace), workspace_bytes, _stream_of(q, stream)))


def a2sf_paged_workspace_bytes(tokens, heads, kv_heads, d, sequences, table_tokens) -> int:
    if max(tokens, heads, kv_heads, d, sequences) > 0x7FFFFFFF:
        return 0
    return int(lib().a2sf_paged_workspace_bytes(tokens, heads, kv_heads, d, sequences, table_tokens))


def _rows_of(x, rows, dtype, like):
    """The C struct of [rows, any] and its columns (None, 0 of None)."""
    if x is None:
        return None, 0
    _reach(x, like)
    _need(x.dim() == 2 and x.shape[0] == rows and (x.stride(1) == 1 or x.shape[1] == 1))
    _need(x.dtype == dtype, A2SF_EDTYPE)
    _int32(x.shape[1])
    return Rows(x.data_ptr(), x.stride(0)), x.shape[1]


def a2sf_log_probs(logits, tokens=None, logp=None, entropy=None, top=None, top_tokens=None, stream=None):
    """tokens [rows, given] int32 with logp [rows, given], entropy [rows], top [rows, alternatives] and top_tokens int32: all but the
    logits may be None."""
    at = _entry("a2sf_log_probs")
    status = _call.log_probs(at, logits, tokens, logp, entropy, top, top_tokens, stream)
    if status >= 0:
        return _check(status)
    _need(logits.dim() == 2)
    rows, n = logits.shape
    _int32(rows, n)
    f = torch.float32
    t, given = _rows_of(tokens, rows, torch.int32, logits)
    l, values = _rows_of(logp, rows, f, logits)
    a, alternatives = _rows_of(top, rows, f, logits)
    i, indices = _rows_of(top_tokens, rows, torch.int32, logits)
    _need(given == values and (top is None or top_tokens is None or alternatives == indices))
    _check(lib().a2sf_log_probs(_rows(logits, logits), rows, n, dtype_code(logits.dtype), t, given, l, _column(entropy, rows, f, logits),
                                a, i, max(alternatives, indices), _stream_of(logits, stream)))
